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
// It is bound by HBM: 4 KiB of keys read and 512 bytes written a block and head (16-bit TARGET).
// A wave's loads depend on its table entries, one round trip a pair; up to 32 waves a compute
// unit, 8 KiB each, cover that.
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
// The ordered form of two words, and back; of bytes and nibbles: BITS below the sign of each element.
__device__ __forceinline__ uint32_t turn_words(uint32_t w, uint32_t mask) {
  return w ^ (__builtin_bit_cast(uint32_t, __builtin_bit_cast(s16x2, w) >> 15) & mask);
}
__device__ __forceinline__ uint32_t turn_bytes(uint32_t w) {
  const uint32_t sign = (w >> 7) & 0x01010101u;
  return w ^ ((sign << 7) - sign);
}
__device__ __forceinline__ uint32_t turn_nibbles(uint32_t w) {
  const uint32_t sign = (w >> 3) & 0x11111111u;
  return w ^ ((sign << 3) - sign);
}
template <int N>
__device__ __forceinline__ uint32_t up(uint32_t w) {
  return __builtin_bit_cast(uint32_t, (u16x2)(__builtin_bit_cast(u16x2, w) << (unsigned short)N));
}

struct Extremes {
  uint32_t low[4], high[4];   // 8 channels, two a register
};

// The 16-bit elements of a row that a lane holds, in ordered form, 8 in all: words as they lie;
// bytes (2 registers) as elements (0, 2), (1, 3), (4, 6), (5, 7); nibbles (1) as (0, 4), (1, 5), (2, 6), (3, 7).
enum Form { kWords, kBytes, kNibbles };

template <int FORM>
__device__ __forceinline__ void ordered(u32x4 w, uint32_t (&x)[4]) {
  if constexpr (FORM == kWords) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = turn_words(w[i], 0x7FFF7FFFu);
  } else if constexpr (FORM == kBytes) {
    const uint32_t a = turn_bytes(w[0]), b = turn_bytes(w[1]);
    x[0] = up<8>(a);
    x[1] = a;
    x[2] = up<8>(b);
    x[3] = b;
  } else {
    const uint32_t a = turn_nibbles(w[0]);
    x[0] = up<12>(a);
    x[1] = up<8>(a);
    x[2] = up<4>(a);
    x[3] = a;
  }
}

// Back to 8 executed words in the order of the elements.
template <int FORM>
__device__ __forceinline__ u32x4 executed(const uint32_t (&x)[4]) {
  if constexpr (FORM == kWords) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = turn_words(x[i], 0x7FFF7FFFu);
    return w;
  } else {
    constexpr uint32_t kKeep = FORM == kBytes ? 0xFF00FF00u : 0xF000F000u, kMask = FORM == kBytes ? 0x7F007F00u : 0x70007000u;
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = turn_words(x[i] & kKeep, kMask);
    constexpr uint32_t kLow = 0x05040100u, kHigh = 0x07060302u;   // (both low halves), (both high halves)
    if constexpr (FORM == kBytes) return u32x4{perm(y[1], y[0], kLow), perm(y[1], y[0], kHigh), perm(y[3], y[2], kLow), perm(y[3], y[2], kHigh)};
    else return u32x4{perm(y[1], y[0], kLow), perm(y[3], y[2], kLow), perm(y[1], y[0], kHigh), perm(y[3], y[2], kHigh)};
  }
}

// min or max over the four lanes that hold the same channels (l, l ^ 16, l ^ 32, l ^ 48)
template <bool HIGH>
__device__ __forceinline__ uint32_t joined(uint32_t x) {
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  const uint32_t y = HIGH ? high2(a[0], a[1]) : low2(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return HIGH ? high2(b[0], b[1]) : low2(b[0], b[1]);
}

// A lane's 8 channels of row 4 r + lane / 16 of a tile whose rows are `row` bytes.
template <int FORM>
__device__ __forceinline__ void load_rows(const char* tile, int lane, u32x4 (&w)[4]) {
  constexpr int kRow = FORM == kWords ? 2 * kHeadDim : (FORM == kBytes ? kHeadDim : kHeadDim / 2);
  const char* p = tile + (lane >> 4) * kRow + (lane & 15) * (kRow / 16);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const char* at = p + 4 * r * kRow;
    if constexpr (FORM == kWords) w[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
    else if constexpr (FORM == kBytes) w[r].xy = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(at));
    else w[r].x = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(at));
  }
}

// The bounds of the `live` first rows, as executed words: the smallest in lanes of even row groups, the largest in odd ones.
template <int FORM>
__device__ __forceinline__ u32x4 reduce(const u32x4 (&w)[4], int live, int lane) {
  Extremes e;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e.low[i] = 0x7FFF7FFFu;
    e.high[i] = 0x80008000u;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    uint32_t x[4];
    ordered<FORM>(w[r], x);
    if (live == kPage) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e.low[i] = low2(e.low[i], x[i]);
        e.high[i] = high2(e.high[i], x[i]);
      }
    } else if (4 * r + (lane >> 4) < live) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e.low[i] = low2(e.low[i], x[i]);
        e.high[i] = high2(e.high[i], x[i]);
      }
    }
  }
  uint32_t out[4];
  const bool high = lane & 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = joined<false>(e.low[i]), b = joined<true>(e.high[i]);
    out[i] = high ? b : a;
  }
  return executed<FORM>(out);
}

__device__ __forceinline__ int clamped(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Wave w takes the w-th equal share of the units: (sequence, KV head, pair of blocks with at least one
// changed block), in this order.
template <bool F8, bool ELASTIC>
__global__ __launch_bounds__(64 * kWaves) void key_bounds_kernel(BoundsArgs a) {
  constexpr int kTile = F8 ? kTileBytes / 2 : kTileBytes, kElem = F8 ? 1 : 2;
  const BlockRows& b = a.rows;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hkv = b.num_kv_heads;
  auto length = [&](int s) { return s < b.batch ? clamped(b.lens[s], 0, b.len_cap) : 0; };
  auto first_block = [&](int s) { return a.known && s < b.batch ? max(a.known[s], 0) / kPage : 0; };
  auto pairs = [&](int s) {   // with a changed block
    const int blocks = (length(s) + kPage - 1) / kPage, from = first_block(s);
    return from < blocks ? (blocks + 1) / 2 - from / 2 : 0;
  };
  int mine = 0;
#pragma unroll 1
  for (int s = lane; s < b.batch; s += 64) mine += pairs(s);
  const int64_t units = (int64_t)last_lane(sum_scan(mine)) * hkv, waves = (int64_t)gridDim.x * kWaves;
  const int64_t id = (int64_t)blockIdx.x * kWaves + wave;
  int64_t u = units * id / waves;
  const int64_t end = units * (id + 1) / waves;
  if (u >= end) return;

  // the sequence of unit u
  int s = 0, np = 0;
  int64_t seq = 0;   // its first unit
  {
    int cum = 0;
#pragma unroll 1
    for (int c0 = 0;; c0 += 64) {
      const int x = pairs(c0 + lane), incl = sum_scan(x);
      const uint64_t hit = __builtin_amdgcn_ballot_w64((int64_t)(cum + incl) * hkv > u);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        s = c0 + l;
        np = __builtin_amdgcn_readlane(x, l);
        seq = (int64_t)(cum + __builtin_amdgcn_readlane(incl, l) - np) * hkv;
        break;
      }
      cum += last_lane(incl);
    }
  }
  int kvh = (int)((u - seq) / np), j = (int)(u - seq) - kvh * np;

  while (true) {
    const int len = length(s), from = first_block(s), blocks = (len + kPage - 1) / kPage;
    int base_lo = 0, base_hi = 0;
    bool by_tags = ELASTIC && b.tags;
    if (ELASTIC && b.base && b.base[2 * s] >= 0) {
      by_tags = false;
      base_lo = 2 * b.base[2 * s];
      base_hi = 2 * b.base[2 * s + 1];
    }
    for (; kvh < hkv; ++kvh, j = 0) {
      for (; j < np; ++j) {
        // both blocks' loads first, then both reductions
        const int i0 = 2 * (from / 2 + j);
        u32x4 w[2][4];
        bool base[2], changed[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const int i = i0 + m;
          changed[m] = i >= from && i < blocks;
          base[m] = false;
          if (!changed[m]) continue;
          const size_t at = (size_t)s * b.max_blocks + i;
          const int entry = b.bt[at], phys = (unsigned)entry < (unsigned)b.num_blocks ? entry : 0;   // never leave the pool
          if constexpr (ELASTIC) base[m] = by_tags ? b.tags[at] != 0 : (i >= base_lo && i < base_hi);
          const char* tile = reinterpret_cast<const char*>(b.pool) + ((size_t)phys * 2 * hkv + kvh) * kTile;
          if (base[m]) load_rows<F8 ? kNibbles : kBytes>(tile + m * (kTile / 2), lane, w[m]);
          else load_rows<F8 ? kBytes : kWords>(tile, lane, w[m]);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          if (!changed[m]) continue;
          const int live = min(kPage, len - (i0 + m) * kPage);
          const u32x4 x = base[m] ? reduce<F8 ? kNibbles : kBytes>(w[m], live, lane) : reduce<F8 ? kBytes : kWords>(w[m], live, lane);
          if (lane < 32) {
            char* dst = static_cast<char*>(a.bounds) +
                        (((size_t)s * hkv + kvh) * b.max_blocks + (i0 + m)) * (2 * kHeadDim * kElem) + lane * 8 * kElem;
            if constexpr (F8)
              *reinterpret_cast<u32x2*>(dst) = u32x2{perm(x[1], x[0], 0x07050301u), perm(x[3], x[2], 0x07050301u)};   // the high bytes
            else
              *reinterpret_cast<u32x4*>(dst) = x;
          }
        }
        if (++u == end) return;
      }
    }
    kvh = j = 0;
    do {   // the next sequence with a changed block (one exists: u < end)
      ++s;
      np = pairs(s);
    } while (np == 0);
  }
}

}  // namespace

hipError_t launch_key_bounds(const BoundsArgs& a, int dtype, bool elastic, hipStream_t st) {
  if (a.rows.batch == 0) return hipSuccess;
  // at most the pairs there can be, and 32 waves a compute unit
  const int64_t most = (int64_t)a.rows.batch * a.rows.num_kv_heads * ((a.rows.len_cap + 2 * kPage - 1) / (2 * kPage));
  const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>((most + kWaves - 1) / kWaves, 2048))), block(64 * kWaves);
  const bool f8 = dtype == 3;
  if (f8 && elastic) hipLaunchKernelGGL((key_bounds_kernel<true, true>), grid, block, 0, st, a);
  else if (f8) hipLaunchKernelGGL((key_bounds_kernel<true, false>), grid, block, 0, st, a);
  else if (elastic) hipLaunchKernelGGL((key_bounds_kernel<false, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((key_bounds_kernel<false, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace ekv
