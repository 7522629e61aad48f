// Bounds of the keys of each block: for every channel of a KV head the smallest and the
// largest executed key over the block's tokens.
//
// A wave takes a pair of blocks of one (sequence, KV head): 16 lanes a row, 8 channels a
// lane, four rows a load, and joins the four row groups at the end.  Keys are
// compared as 16-bit integers that order as the values do (a word's lower bits turned over
// where its sign is set): two channels an instruction, -0 below 0, and a NaN beyond the
// infinity of its sign, so that no rounding takes place and a NaN is not lost.  Bytes and nibbles are compared
// in the upper bits of such integers, with whatever lies below them left in place (it only decides between equals).
//
// It is bound by HBM: 4 KiB of keys read and 512 bytes written a block and head (16-bit TARGET).  Prompts of
// 164 thousand 16-bit tokens, 8 KV heads: 81 us (417 MB, 5.1 TB/s); 600 thousand 8-bit ones, half of them BASE, 117 us
// (518 MB, 4.4 TB/s: vector work for nibbles and bytes is half of the time); one token of 64 sequences 4.0 us, a launch.
#include <algorithm>

#include "common.h"
#include "long_context.h"
#include "wave_scan.h"

namespace ekv {
namespace {

constexpr int kWaves = 4;

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t low2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
}
__device__ __forceinline__ uint32_t high2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
}
// The ordered form of two words (bytes: in their upper halves), and back; of 8 nibbles.
__device__ __forceinline__ uint32_t turn_words(uint32_t w, uint32_t mask) {
  return w ^ (__builtin_bit_cast(uint32_t, __builtin_bit_cast(s16x2, w) >> 15) & mask);
}
__device__ __forceinline__ uint32_t turn_nibbles(uint32_t w) {
  const uint32_t sign = (w >> 3) & 0x11111111u;
  uint32_t up = sign << 3;
  asm("" : "+v"(up));   // (else the two become a multiplication, four times as slow as both)
  return w ^ (up - sign);
}
template <int N>
__device__ __forceinline__ uint32_t up(uint32_t w) {
  return __builtin_bit_cast(uint32_t, (u16x2)(__builtin_bit_cast(u16x2, w) << (unsigned short)N));
}

// The 16-bit elements of a row that a lane holds, in ordered form, 8 in all: words as they lie;
// bytes (2 registers) as elements (0, 2), (1, 3), (4, 6), (5, 7); nibbles (1) as (0, 4), (1, 5), (2, 6), (3, 7).
enum Form { kWords, kBytes, kNibbles };

template <int FORM>
__device__ __forceinline__ void ordered(u32x4 w, uint32_t (&x)[4]) {
  if constexpr (FORM == kWords) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = turn_words(w[i], 0x7FFF7FFFu);
  } else if constexpr (FORM == kBytes) {
    x[0] = turn_words(up<8>(w[0]), 0x7FFF7FFFu);
    x[1] = turn_words(w[0], 0x7FFF7FFFu);
    x[2] = turn_words(up<8>(w[1]), 0x7FFF7FFFu);
    x[3] = turn_words(w[1], 0x7FFF7FFFu);
  } else {
    const uint32_t a = turn_nibbles(w[0]);
    x[0] = up<12>(a);
    x[1] = up<8>(a);
    x[2] = up<4>(a);
    x[3] = a;
  }
}

// Four registers of extremes, joined over the lanes that hold the same channels (l, l ^ 16, l ^ 32, l ^ 48) and dealt out
// to them: row group r of lanes gets elements 2 r, 2 r + 1, as executed words.
template <int FORM, bool HIGH>
__device__ __forceinline__ uint32_t joined(const uint32_t (&x)[4]) {
  constexpr uint32_t kLow = 0x05040100u, kUp = 0x07060302u;   // (both low halves), (both high halves)
  uint32_t y[4];
  if constexpr (FORM == kWords) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = x[i];
  } else if constexpr (FORM == kBytes) {
    y[0] = perm(x[1], x[0], kLow);
    y[1] = perm(x[1], x[0], kUp);
    y[2] = perm(x[3], x[2], kLow);
    y[3] = perm(x[3], x[2], kUp);
  } else {
    y[0] = perm(x[1], x[0], kLow);
    y[1] = perm(x[3], x[2], kLow);
    y[2] = perm(x[1], x[0], kUp);
    y[3] = perm(x[3], x[2], kUp);
  }
  auto pick = [](uint32_t a, uint32_t b) { return HIGH ? high2(a, b) : low2(a, b); };
  const auto a = __builtin_amdgcn_permlane16_swap(y[0], y[1], false, false);
  const auto b = __builtin_amdgcn_permlane16_swap(y[2], y[3], false, false);
  const auto c = __builtin_amdgcn_permlane32_swap(pick(a[0], a[1]), pick(b[0], b[1]), false, false);
  constexpr uint32_t kKeep = FORM == kWords ? 0xFFFFFFFFu : (FORM == kBytes ? 0xFF00FF00u : 0xF000F000u);
  return turn_words(pick(c[0], c[1]) & kKeep, kKeep & 0x7FFF7FFFu);
}

// What a lane loads of a row: its 8 channels as words (16 bytes), or bytes (8).  Of a BASE row, half as wide, it
// loads as much, at a multiple of that, and takes its half: the number of loads in flight does
// not depend on the mode, so waits count them exactly.
template <bool F8> struct Lane;
template <> struct Lane<false> {
  typedef u32x4 row;
  static __device__ __forceinline__ u32x4 base(u32x4 w, bool odd) { return u32x4{odd ? w.z : w.x, odd ? w.w : w.y, 0u, 0u}; }
  static __device__ __forceinline__ u32x4 target(u32x4 w) { return w; }
};
template <> struct Lane<true> {
  typedef u32x2 row;
  static __device__ __forceinline__ u32x4 base(u32x2 w, bool odd) { return u32x4{odd ? w.y : w.x, 0u, 0u, 0u}; }
  static __device__ __forceinline__ u32x4 target(u32x2 w) { return u32x4{w.x, w.y, 0u, 0u}; }
};

// The bounds of the `live` first rows: lane (r, l) = (lane / 16, lane % 16) gets elements 8 l + 2 r, + 1, as executed words.
template <int FORM, bool F8>
__device__ __forceinline__ void reduce(const typename Lane<F8>::row (&w)[4], int live, int lane, uint32_t& low, uint32_t& high) {
  constexpr bool kTarget = FORM == (F8 ? kBytes : kWords);
  uint32_t x[4][4];
#pragma unroll
  for (int r = 0; r < 4; ++r) ordered<FORM>(kTarget ? Lane<F8>::target(w[r]) : Lane<F8>::base(w[r], lane & 1), x[r]);
  uint32_t lo[4], hi[4];
  if (live == kPage) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = low2(low2(x[0][i], x[1][i]), low2(x[2][i], x[3][i]));
      hi[i] = high2(high2(x[0][i], x[1][i]), high2(x[2][i], x[3][i]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = 0x7FFF7FFFu;
      hi[i] = 0x80008000u;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const bool counts = 4 * r + (lane >> 4) < live;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = low2(lo[i], counts ? x[r][i] : 0x7FFF7FFFu);
        hi[i] = high2(hi[i], counts ? x[r][i] : 0x80008000u);
      }
    }
  }
  low = joined<FORM, false>(lo);
  high = joined<FORM, true>(hi);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }   // (the same in all lanes)
__device__ __forceinline__ int clamped(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Wave w takes the w-th equal share of the units: (sequence, pair of blocks with at least one changed
// block, KV head), in this order, so that a pair's table entries serve all heads and its tiles lie side by side.  A
// unit's loads go out before the one before it is reduced.
template <bool F8, bool ELASTIC>
__global__ __launch_bounds__(64 * kWaves) void key_bounds_kernel(BoundsArgs a) {
  constexpr int kTile = F8 ? kTileBytes / 2 : kTileBytes, kElem = F8 ? 1 : 2;
  typedef typename Lane<F8>::row Row;
  const BlockRows& b = a.rows;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hkv = b.num_kv_heads;
  // Lane l: length and first changed block of sequence window + l.
  int window = 0, len_lane = 0, from_lane = 0;
  auto read_lengths = [&](int c0) {
    window = c0;
    len_lane = from_lane = 0;
    if (c0 + lane < b.batch) {
      const int length = b.lens[c0 + lane], known = (a.known ? a.known : b.lens)[c0 + lane];   // (one round trip)
      len_lane = clamped(length, 0, b.len_cap);
      from_lane = a.known ? max(known, 0) / kPage : 0;
    }
  };
  auto pairs_lane = [&]() {   // with a changed block
    const int blocks = (len_lane + kPage - 1) / kPage;
    return from_lane < blocks ? (blocks + 1) / 2 - from_lane / 2 : 0;
  };
  read_lengths(0);
  int mine = pairs_lane();
  const int first_pairs = mine;
#pragma unroll 1
  for (int c0 = 64; c0 < b.batch; c0 += 64) {
    read_lengths(c0);
    mine += pairs_lane();
  }
  const uint32_t units = (uint32_t)last_lane(sum_scan(mine)) * hkv, waves = gridDim.x * kWaves, id = blockIdx.x * kWaves + wave;
  const uint32_t share = units / waves, extra = units - share * waves;   // (the first `extra` waves take one more)
  const uint32_t begin = id * share + min(id, extra), end = begin + share + (id < extra ? 1 : 0);
  if (begin >= end) return;

  // A sequence, and the position in it of the unit whose loads go out next.
  int s = 0, np = 0, j = 0, kvh = 0, len = 0, from = 0;
  {
    uint32_t cum = 0;
#pragma unroll 1
    for (int c0 = 0;; c0 += 64) {
      if (c0 != window) read_lengths(c0);
      const int x = c0 == 0 ? first_pairs : pairs_lane(), incl = sum_scan(x);
      const uint64_t hit = __builtin_amdgcn_ballot_w64((cum + incl) * hkv > begin);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        s = uniform(c0 + l);
        np = __builtin_amdgcn_readlane(x, l);
        const uint32_t off = begin - (cum + __builtin_amdgcn_readlane(incl, l) - np) * hkv;
        j = uniform(off / hkv);
        kvh = uniform(off - j * hkv);
        break;
      }
      cum += last_lane(incl);
    }
  }
  int base_lo, base_hi;
  bool by_tags;
  auto enter = [&]() {
    len = uniform(__builtin_amdgcn_readlane(len_lane, s - window));
    from = uniform(__builtin_amdgcn_readlane(from_lane, s - window));
    base_lo = base_hi = 0;
    by_tags = ELASTIC && b.tags;
    if (ELASTIC && b.base) {
      const int p0 = b.base[2 * s], p1 = b.base[2 * s + 1];
      if (p0 >= 0) {
        by_tags = false;
        base_lo = 2 * p0;
        base_hi = 2 * p1;
      }
    }
  };
  // Lane l: physical block l of the 32 pairs from pair `entries` on, with its tag in the sign.
  int entries = 0, entry_lane = 0;
  auto read_entries = [&]() {
    entries = j;
    const int i = 2 * (from / 2 + j) + lane;
    entry_lane = 0;
    if (i * kPage < len) {
      const size_t at = (size_t)s * b.max_blocks + i;
      const int entry = b.bt[at];
      const uint8_t tag = (by_tags ? b.tags : reinterpret_cast<const uint8_t*>(b.bt))[at];   // (one round trip)
      entry_lane = (unsigned)entry < (unsigned)b.num_blocks ? entry : 0;   // never leave the pool
      if (ELASTIC && by_tags && tag != 0) entry_lane |= 1 << 31;
    }
  };
  enter();
  read_entries();

  // A unit on its way: where its bounds go, and of each block the tokens that count (0: not changed) and the mode.
  struct Unit {
    Row w[2][4];
    size_t to;
    int live[2];
    bool base[2];
  };
  // of the current pair of the sequence, as entered at its first head
  const char* tile[2];
  int live[2];
  bool base[2];
  uint32_t off[2], step[2];
  const uint32_t target_row = kHeadDim * kElem, base_row = target_row / 2;
  const uint32_t target_off = (lane >> 4) * target_row + (lane & 15) * (target_row / 16),
                 base_off = (lane >> 4) * base_row + (lane & 14) * (base_row / 16);
  auto enter_pair = [&]() {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int i = uniform(2 * (from / 2 + j) + m), at = uniform(2 * (j - entries) + m);
      const bool changed = i >= uniform(from) && i * kPage < uniform(len);   // (one of the two is; the other's loads go to any block)
      const int entry = __builtin_amdgcn_readlane(entry_lane, at);
      live[m] = changed ? min(kPage, uniform(len) - i * kPage) : 0;
      base[m] = ELASTIC && changed && (by_tags ? entry < 0 : (i >= base_lo && i < base_hi));
      tile[m] = reinterpret_cast<const char*>(b.pool) + (size_t)(entry & 0x7FFFFFFF) * 2 * hkv * kTile + (base[m] ? m * (kTile / 2) : 0);
      off[m] = base[m] ? base_off : target_off;
      step[m] = base[m] ? 4 * base_row : 4 * target_row;
    }
  };
  enter_pair();
  auto load = [&](Unit& u) {   // the unit at (s, j, kvh); then moves on
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const char* src = tile[m] + (size_t)kvh * kTile;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        uint32_t at = off[m] + r * step[m];
        asm volatile("" : "+v"(at));   // (opaque: the load then takes a scalar base and this offset)
        // (past the caches, which the bounds have to themselves: those prompts 81.5 us, through them 90.2)
        u.w[m][r] = __builtin_nontemporal_load(reinterpret_cast<const Row*>(src + at));
      }
      u.live[m] = live[m];
      u.base[m] = base[m];
    }
    u.to = (((size_t)s * hkv + kvh) * b.max_blocks + 2 * (from / 2 + j)) * (2 * kHeadDim * kElem);
  };
  auto advance = [&]() {
    if (++kvh < hkv) return;
    kvh = 0;
    j = uniform(j + 1);
    if (j == uniform(np)) {
      j = 0;
      uint64_t hit;
      int x;
      ++s;
      while (true) {   // the next sequence with a changed block (one exists while units are left)
        if (s - window >= 64) read_lengths(s);
        x = pairs_lane();
        hit = __builtin_amdgcn_ballot_w64(x > 0 && lane >= s - window);
        if (hit) break;
        s = window + 64;
      }
      s = uniform(window + __builtin_ctzll(hit));
      np = __builtin_amdgcn_readlane(x, s - window);
      enter();
      read_entries();
    } else if (uniform(j - entries) == 32) {
      read_entries();
    }
    enter_pair();
  };
  auto finish = [&](const Unit& u) {   // (blocks that are not changed are reduced too: what was loaded has to be waited for)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      uint32_t low, high;
      if (ELASTIC && u.base[m]) reduce<F8 ? kNibbles : kBytes, F8>(u.w[m], u.live[m], lane, low, high);
      else reduce<F8 ? kBytes : kWords, F8>(u.w[m], u.live[m], lane, low, high);
      if (u.live[m] > 0) {
        char* dst = static_cast<char*>(a.bounds) + u.to + m * (2 * kHeadDim * kElem) + (8 * (lane & 15) + 2 * (lane >> 4)) * kElem;
        if constexpr (F8) {   // the high bytes
          *reinterpret_cast<uint16_t*>(dst) = (uint16_t)perm(0u, low, 0x0C0C0301u);
          *reinterpret_cast<uint16_t*>(dst + kHeadDim) = (uint16_t)perm(0u, high, 0x0C0C0301u);
        } else {
          *reinterpret_cast<uint32_t*>(dst) = low;
          *reinterpret_cast<uint32_t*>(dst + 2 * kHeadDim) = high;
        }
      }
    }
  };
  Unit one, two;
  load(one);
#pragma unroll 1
  for (uint32_t u = begin;; u += 2) {   // (the last unit is loaded again rather than none: the loads stay countable)
    if (u + 1 < end) advance();
    load(two);
    finish(one);
    if (u + 1 >= end) return;
    if (u + 2 < end) advance();
    load(one);
    finish(two);
    if (u + 2 >= end) return;
  }
}

}  // namespace

hipError_t launch_key_bounds(const BoundsArgs& a, int dtype, bool elastic, hipStream_t st) {
  if (a.rows.batch == 0) return hipSuccess;
  // As many workgroups as there can be pairs of blocks, at most two waves a SIMD, of 8-bit pools, whose units are half as
  // many bytes, four: 164 thousand 16-bit tokens of 8 heads 81.5 us (four waves: 84.0, eight, in turn: 88.1), 600 thousand
  // 8-bit ones, half of them BASE, 117 (two waves: 125).
  const bool f8 = dtype == 3;
  const int64_t most = (int64_t)a.rows.batch * a.rows.num_kv_heads * ((a.rows.len_cap + 2 * kPage - 1) / (2 * kPage));
  const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>((most + kWaves - 1) / kWaves, f8 ? 1024 : 512))), block(64 * kWaves);
  if (f8 && elastic) hipLaunchKernelGGL((key_bounds_kernel<true, true>), grid, block, 0, st, a);
  else if (f8) hipLaunchKernelGGL((key_bounds_kernel<true, false>), grid, block, 0, st, a);
  else if (elastic) hipLaunchKernelGGL((key_bounds_kernel<false, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((key_bounds_kernel<false, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace ekv
