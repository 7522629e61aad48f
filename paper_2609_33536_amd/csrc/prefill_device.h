// Device building blocks of the attention kernels that work on 32-key units and
// 32 query columns per wave (internal header): the unit's place in LDS, its
// loads and widening, the block table in lane registers, and the online softmax
// on 32x32x16 matrix cores.  prefill.hip describes the lane layout.
#pragma once

#include "attn_device.h"

namespace ekv {
namespace {

constexpr int kPfCols = 32;       // query columns per wave
constexpr int kPfWindow = 64;     // pairs per metadata window: one per lane

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4v* lds_i16x4;

template <typename T> struct Mma32;
template <> struct Mma32<Bf16> {
  static __device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b),
                                                   c, 0, 0, 0);
  }
};
template <> struct Mma32<Fp16> {
  static __device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b),
                                                  c, 0, 0, 0);
  }
};

// Two probabilities -> packed 16-bit heads and packed 16-bit remainders
// (head + remainder = p to ~16 significant bits).  bf16: the head is the
// upper half of the fp32 word (truncation), one byte permute for the pair.
template <typename T>
__device__ __forceinline__ void split_p(float p0, float p1, uint32_t& hi, uint32_t& lo);

template <>
__device__ __forceinline__ void split_p<Bf16>(float p0, float p1, uint32_t& hi, uint32_t& lo) {
  const uint32_t x0 = __float_as_uint(p0), x1 = __float_as_uint(p1);
  hi = perm(x1, x0, 0x07060302u);   // upper halves: x0 -> low word, x1 -> high word
  // both remainders rounded to nearest-even in one packed conversion
  const f32x2v rem = {p0 - __uint_as_float(x0 & 0xffff0000u), p1 - __uint_as_float(x1 & 0xffff0000u)};
  lo = __builtin_bit_cast(uint32_t, __builtin_convertvector(rem, bf16x2v));
}
template <>
__device__ __forceinline__ void split_p<Fp16>(float p0, float p1, uint32_t& hi, uint32_t& lo) {
  // one packed conversion for the heads (to nearest); p - head is exact, so one
  // mixed-precision fused multiply-add rounds each remainder into its half
  typedef _Float16 f16x2v __attribute__((ext_vector_type(2)));
  const f16x2v h = __builtin_convertvector((f32x2v{p0, p1}), f16x2v);
  const f16x2v r = {(_Float16)__builtin_fmaf(-1.0f, (float)h[0], p0), (_Float16)__builtin_fmaf(-1.0f, (float)h[1], p1)};
  hi = __builtin_bit_cast(uint32_t, h);
  lo = __builtin_bit_cast(uint32_t, r);
}

// 8 nibbles (element e in byte e/2, low nibble for even e) -> 8 bytes,
// each nibble in the high half of its byte (an executed 4-bit BASE value).
__device__ __forceinline__ u32x2 widen_nibbles(uint32_t w) {
  const uint32_t even = (w << 4) & 0xF0F0F0F0u, odd = w & 0xF0F0F0F0u;
  return u32x2{perm(odd, even, 0x05010400u), perm(odd, even, 0x07030602u)};
}

// max of three floats.  Written for the compiler, not as inline assembly:
// its operands come straight from the matrix cores, and only the compiler
// inserts the wait states a vector instruction needs before it may read an
// MFMA result (inline assembly would read the registers while the products
// are still being written).
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_fmaxf(__builtin_fmaxf(a, b), c); }

// v *= f, written for the compiler: the accumulators come straight from the
// matrix cores, and only the compiler inserts the wait states a vector
// instruction needs before it reads an MFMA result.  (On gfx950 the
// multiplies stay in the accumulators' own registers: no copies on the
// common path that skips the rescale.)
__device__ __forceinline__ void scale_in_place(f32x16& v, float f) {
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] *= f;
}

// Workgroup barrier that also orders this wave's LDS accesses.  On gfx950
// s_barrier does not wait for the wave's outstanding LDS operations, and
// the compiler adds no wait before a bare s_barrier: an LDS write issued
// before it (the widened 8-bit tiles) could land after another wave has
// passed the barrier and read the old bytes, and an LDS read still in
// flight could see a slot that the ring's next load has begun to refill.
// s_waitcnt lgkmcnt(0) completes every LDS access of the wave first.  The
// ring's direct-to-LDS loads are vector memory operations, waited for with
// explicit counts before the barrier that publishes a slot.
__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A unit's slot in LDS: the K rows of both blocks, then the V rows, in groups
// of 4 rows: 1 KiB (one direct-to-LDS load: 64 lanes x 16 bytes) and 16 bytes
// of padding.  In a group, 16-byte chunk c of row r sits at position
// 16 (c / 4) + 4 r + c % 4.  So a K read (16 rows, one chunk) and a transposing
// V read (4 rows x 4 chunks of one group) touch 16 distinct 16-byte positions
// of a 256-byte bank cycle, and the head-dim step, the dim tile and the key
// step of every read are constant offsets from one address per lane.
constexpr int kGroup = 1024 + 16;
constexpr int kTilePf = 4 * kGroup;       // 16 rows
constexpr int kSlotPf = 4 * kTilePf;      // K of both blocks, V of both
constexpr int kPlanePf = 2 * kTilePf;     // V's offset in a slot

// Offset of row group 2 half of block `member`: quarter q = 2 member + half of
// a plane, 8 rows, is loaded and widened as one piece.
__device__ __forceinline__ constexpr uint32_t quarter_offset(int q) { return (q >> 1) * kTilePf + 2 * (q & 1) * kGroup; }

// One direct-to-LDS load: lane l's 16 bytes at base + off go to lds + 16 l.
// Inline assembly (it writes no register) keeps it out of the compiler's wait
// insertion, which would wait for every load in flight before each transposing
// LDS read; the kernels wait with explicit counts.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // (m0 is named as clobbered although the compiler never allocates it)
__device__ __forceinline__ void dma16(uint64_t base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Loads and widening of quarters.  A unit costs a quarter kLoads loads (2 of
// K, 2 of V; half for 8-bit pools) whatever its kind, so that constant counts
// wait for it: a 16-bit BASE quarter has half the bytes and loads them twice
// (the copy is overwritten when the quarter is widened), an 8-bit BASE quarter
// of 512 bytes twice with the two halves of the wave.
template <bool F8>
struct Stager {
  static constexpr int kLoads = F8 ? 2 : 4;
  static constexpr int kTileP = F8 ? kTileBytes / 2 : kTileBytes;   // a (plane, head) tile in the pool
  uint32_t src_t, src_b, src_n;   // source offsets in a quarter: words, bytes, nibbles
  uint32_t raw_n, dst;            // nibbles' place in the raw quarter; this lane's words in the widened one
  int row;                        // row of the quarter whose 16-element chunk this lane widens
  uint64_t v_off;                 // K plane -> V plane in the pool

  __device__ __forceinline__ Stager(int lane, int num_kv_heads) {
    src_t = ((lane >> 2) & 3) * 256 + 64 * (lane >> 4) + 16 * (lane & 3);
    // lane -> (row, chunk) so that 16 consecutive lanes write 16 distinct
    // positions of a bank cycle when they widen
    row = (lane >> 1) & 7;
    const int chunk = 2 * (lane >> 4) + (lane & 1);
    src_b = row * kHeadDim + 16 * chunk;
    src_n = 16 * (lane & 31);
    raw_n = row * (kHeadDim / 2) + 8 * chunk;
    dst = (row >> 2) * kGroup + 256 * (chunk >> 1) + 64 * (row & 3) + 32 * (chunk & 1);
    v_off = (uint64_t)num_kv_heads * kTileP;
  }
  // Quarter q of a unit, its two planes to places of their own (K first: kLoads / 2 loads
  // each).  tile: the K tile of the quarter's block (a BASE pair's: the packed tile).
  __device__ __forceinline__ void load_planes(uint64_t tile, bool base, int q, uint32_t k_slot, uint32_t v_slot) const {
    const uint32_t at = quarter_offset(q);
    const uint64_t packed = tile + (uint32_t)(q >> 1) * (kTileP / 2);
    if constexpr (F8) {
      const uint32_t off = base ? src_n : src_b;
      const uint64_t src = base ? packed + (q & 1) * 8 * (kHeadDim / 2) : tile + (q & 1) * 8 * kHeadDim;
      dma16(src, off, k_slot + at);
      dma16(src + v_off, off, v_slot + at);
    } else {
      const uint32_t off = base ? src_b : src_t;
      const uint64_t src = base ? packed + (q & 1) * 8 * kHeadDim : tile + (q & 1) * 8 * 2 * kHeadDim;
      const uint64_t src2 = src + (base ? 0 : 1024);
      dma16(src, off, k_slot + at);
      dma16(src2, off, k_slot + at + kGroup);
      dma16(src + v_off, off, v_slot + at);
      dma16(src2 + v_off, off, v_slot + at + kGroup);
    }
  }
  // ... to the unit's slot (LDS address).
  __device__ __forceinline__ void load(uint64_t tile, bool base, int q, uint32_t slot) const {
    load_planes(tile, base, q, slot, slot + kPlanePf);
  }
  // After quarter q of a plane has landed: what landed, and bytes or nibbles -> words in
  // place (by one wave, all of whose reads precede its writes).
  __device__ __forceinline__ u32x4 landed_plane(const char* slot, bool base, int q, int lane) const {
    const char* at = slot + quarter_offset(q);
    if (!F8 && !base) return u32x4{0u, 0u, 0u, 0u};
    if (F8 && base) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(at + raw_n);
      return u32x4{x.x, x.y, 0u, 0u};
    }
    return *reinterpret_cast<const u32x4*>(at + 16 * lane);
  }
  __device__ __forceinline__ void widen_plane(char* slot, bool base, int q, u32x4 raw) const {
    if (!F8 && !base) return;
    char* at = slot + quarter_offset(q);
    if (F8 && base) {
      const u32x2 lo = widen_nibbles(raw.x), hi = widen_nibbles(raw.y);
      raw = u32x4{lo.x, lo.y, hi.x, hi.y};
    }
    *reinterpret_cast<u32x4*>(at + dst) = expand_base8(raw.xy);
    *reinterpret_cast<u32x4*>(at + dst + 16) = expand_base8(raw.zw);
  }
  // Zero V rows for keys at or past `valid` (their slots may hold anything, and 0 * NaN
  // would poison the products).  key0: the unit's first key.
  __device__ __forceinline__ void clear_tail(char* v_slot, int q, int key0, int valid) const {
    if (key0 + 2 * kPage > valid && key0 + 8 * q + row >= valid) {
      char* at = v_slot + quarter_offset(q) + dst;
      *reinterpret_cast<u32x4*>(at) = u32x4{0u, 0u, 0u, 0u};
      *reinterpret_cast<u32x4*>(at + 16) = u32x4{0u, 0u, 0u, 0u};
    }
  }
  // Both planes of quarter q of a unit's slot, in one step: under one branch where the two
  // functions above take one each (prefill's code grows by 0.7 % with them).
  __device__ __forceinline__ void widen(char* slot, bool base, int q, int key0, int valid, int lane) const {
    char* at = slot + quarter_offset(q);
    if (F8 || base) {
      u32x4 raw[2];
#pragma unroll
      for (int pl = 0; pl < 2; ++pl) {
        if (F8 && base) {
          const u32x2 x = *reinterpret_cast<const u32x2*>(at + pl * kPlanePf + raw_n);
          const u32x2 lo = widen_nibbles(x.x), hi = widen_nibbles(x.y);
          raw[pl] = u32x4{lo.x, lo.y, hi.x, hi.y};
        } else {
          raw[pl] = *reinterpret_cast<const u32x4*>(at + pl * kPlanePf + 16 * lane);
        }
      }
#pragma unroll
      for (int pl = 0; pl < 2; ++pl) {
        *reinterpret_cast<u32x4*>(at + pl * kPlanePf + dst) = expand_base8(raw[pl].xy);
        *reinterpret_cast<u32x4*>(at + pl * kPlanePf + dst + 16) = expand_base8(raw[pl].zw);
      }
    }
    clear_tail(slot + kPlanePf, q, key0, valid);
  }
};

// The block table of one sequence in windows of 64 pairs: lane l holds the K
// tile addresses of both blocks of pair w0 + l, and a mask the pairs' modes, so
// that a unit's loads read their addresses from a lane, with no LDS or memory
// round trip.  The next window's entries are fetched a window ahead.
template <bool ELASTIC, bool F8>
struct PairTable {
  const int32_t* row;
  const uint8_t* tags;
  int base_lo = 0, base_hi = 0;   // BASE pairs by boundaries (when the tags are not used)
  bool use_tags = false;
  int nblk, units, num_blocks;
  uint64_t pool, block_bytes;
  int w0 = 0;
  uint64_t addr0 = 0, addr1 = 0, base_mask = 0;   // the current window
  int next0 = 0, next1 = 0;                       // the next one, as read
  bool next_base = false;

  // row s of the table of `a` (the fields of PrefillArgs that name the pool, the table and its modes), from unit `first`
  template <typename Args>
  __device__ __forceinline__ PairTable(const Args& a, int s, int kvh, int nblk_, int lane, int first = 0) : nblk(nblk_) {
    row = a.bt + (size_t)s * a.max_blocks;
    tags = a.tags ? a.tags + (size_t)s * a.max_blocks : nullptr;
    units = (nblk + 1) >> 1;
    num_blocks = a.num_blocks;
    block_bytes = (uint64_t)2 * a.num_kv_heads * Stager<F8>::kTileP;
    pool = reinterpret_cast<uint64_t>(a.pool) + (uint64_t)kvh * Stager<F8>::kTileP;
    if constexpr (ELASTIC) {
      int b0 = -1, b1 = -1;
      if (a.bounds) {
        b0 = a.bounds[2 * s];
        b1 = a.bounds[2 * s + 1];
      }
      if (b0 >= 0) {
        base_lo = b0;
        base_hi = b1;
      } else if (tags) {
        use_tags = true;
      }
    }
    w0 = first & ~(kPfWindow - 1);
    fetch(w0, lane);
    enter();
    if (units > w0 + kPfWindow) fetch(w0 + kPfWindow, lane);
  }
  __device__ __forceinline__ void fetch(int from, int lane) {
    const int p = from + lane;
    next0 = next1 = 0;
    next_base = false;
    if (p < units) {
      next0 = row[2 * p];
      next1 = 2 * p + 1 < nblk ? row[2 * p + 1] : next0;   // a lone last block stands in for the missing one (masked)
      if constexpr (ELASTIC) next_base = use_tags ? tags[2 * p] != 0 : (p >= base_lo && p < base_hi);
    }
  }
  __device__ __forceinline__ void enter() {
    const int b0 = (unsigned)next0 < (unsigned)num_blocks ? next0 : 0;   // never leave the pool
    const int b1 = (unsigned)next1 < (unsigned)num_blocks ? next1 : 0;
    addr0 = pool + (uint64_t)(uint32_t)b0 * block_bytes;
    addr1 = next_base ? addr0 : pool + (uint64_t)(uint32_t)b1 * block_bytes;   // (a BASE pair lies in its first block)
    base_mask = __builtin_amdgcn_ballot_w64(next_base);
  }
  // unit u (nondecreasing over calls); its mode
  __device__ __forceinline__ bool seek(int u, int lane) {
    if (u >= w0 + kPfWindow) {
      w0 = u & ~(kPfWindow - 1);
      enter();
      if (w0 + kPfWindow < units) fetch(w0 + kPfWindow, lane);
    }
    return ELASTIC && ((base_mask >> (u & (kPfWindow - 1))) & 1) != 0;
  }
  __device__ __forceinline__ uint64_t tile(int u, int member) const {
    const uint64_t a = member ? addr1 : addr0;
    const int l = u & (kPfWindow - 1);
    uint64_t at = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(a >> 32), l) << 32) |
                  (uint32_t)__builtin_amdgcn_readlane((uint32_t)a, l);
    // A scalar register that a vector instruction writes needs 5 wait states
    // before a vector memory instruction reads it; the hardware does not check,
    // and the compiler does not look into dma16.  These 3, and the 2 before
    // dma16's load, for all the loads that use the address (waiting in every
    // load cost the 8B chunked prefill 1 %).
    asm("s_nop 2" : "+s"(at));
    return at;
  }
};

// One wave's 32 query columns: their queries, limits and softmax state (lane l
// holds column l % 32; lanes l and l ^ 32 share it).
template <typename T>
struct ColumnState {
  u32x4 q[8];              // Q^T operands: dims 16 k + 8 h .. + 7
  size_t row;              // this lane's query row (element offset in q and out)
  int lim, lim_all;        // keys this lane's column sees; keys every column sees
  bool ok;
  float c_scale;           // |scale| log2(e): a negative scale negates the queries instead (exact)
  f32x16 o[4];
  float m = -__builtin_inff(), l = 0.f;   // reference max (log2 units, the same in lanes l and l ^ 32), this lane's sum

  // the queries of this lane's column, from `queries` at element offset `row` (none if !ok)
  __device__ __forceinline__ void load_queries(const uint16_t* queries, float scale_log2, int h) {
    c_scale = fabsf(scale_log2);
    const uint32_t sign = scale_log2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      q[k] = ok ? (*reinterpret_cast<const u32x4*>(queries + row + 16 * k + 8 * h) ^ sign) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = f32x16{};
  }
  __device__ __forceinline__ f32x16 scores(const u32x4 (&k)[8]) const {
    f32x16 s = f32x16{};
#pragma unroll
    for (int i = 0; i < 8; ++i) s = Mma32<T>::mma(k[i], q[i], s);
    return s;
  }
  // Scores enter the softmax as s * c in log2 units (c is returned).  Units
  // that every column sees whole fold c into the max and the exponent; the
  // others scale first and then set masked keys to -inf, so that a zero
  // scale never multiplies an infinity (0 * -inf is NaN).
  __device__ __forceinline__ float mask(f32x16& s, int key0, int h) const {
    if (key0 + 2 * kPage <= lim_all) return c_scale;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      s[r] = key0 + 8 * (r >> 2) + 4 * h + (r & 3) >= lim ? -__builtin_inff() : s[r] * c_scale;
    return 1.0f;
  }
  // Moves the reference max if some column's unit max exceeds it by more than
  // 2^8 (wave-uniform result); then *shift = old - new reference (log2).
  __device__ __forceinline__ bool advance(const f32x16& s, float c, float* shift) {
    const float m0 = max3(s[0], s[1], s[2]), m1 = max3(s[3], s[4], s[5]);
    const float m2 = max3(s[6], s[7], s[8]), m3 = max3(s[9], s[10], s[11]);
    const float m4 = max3(s[12], s[13], s[14]);
    float mx = max3(max3(m0, m1, m2), max3(m3, m4, s[15]), m0);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = __builtin_fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c;
    const bool moved = __builtin_amdgcn_ballot_w64(mx > m + 8.0f) != 0;
    const float to = moved ? __builtin_fmaxf(m, mx) : m;
    *shift = m - to;
    m = to;
    return moved;
  }
  // P = exp2(s c - ref) as 16-bit heads and remainders; returns the lane's sum.
  __device__ __forceinline__ float probabilities(const f32x16& s, float c, float ref, u32x4 (&hi)[2], u32x4 (&lo)[2]) const {
    float sum[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = fast_exp2(__builtin_fmaf(s[8 * ks + i], c, -ref));
      sum[ks] = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      uint32_t wh[4], wl[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) split_p<T>(p[2 * i], p[2 * i + 1], wh[i], wl[i]);
      hi[ks] = u32x4{wh[0], wh[1], wh[2], wh[3]};
      lo[ks] = u32x4{wl[0], wl[1], wl[2], wl[3]};
    }
    return sum[0] + sum[1];
  }
  __device__ __forceinline__ void accumulate(const u32x4 (&v)[4], u32x4 p) {
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = Mma32<T>::mma(v[t], p, o[t]);
  }
  __device__ __forceinline__ void rescale(float f) {
    l *= f;
#pragma unroll
    for (int t = 0; t < 4; ++t) scale_in_place(o[t], f);
  }
  __device__ __forceinline__ float total() const {   // the column's sum
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
};

// Per-lane offsets of the K and V^T reads in a slot.
__device__ __forceinline__ uint32_t k_read_offset(int lane) {
  const int n = lane & 31;   // key row; chunk 2 k + h of step k
  return (n >> 4) * kTilePf + ((n >> 2) & 3) * kGroup + 64 * (n & 3) + 16 * (lane >> 5);
}
__device__ __forceinline__ uint32_t v_read_offset(int lane) {
  const int i = lane & 15, key = i >> 2, d = i & 3;
  return kPlanePf + (lane >> 5) * kGroup + 64 * key + 16 * (2 * ((lane >> 4) & 1) + (d >> 1)) + 8 * (d & 1);
}
__device__ __forceinline__ void read_k(const char* at, u32x4 (&k)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) k[i] = *reinterpret_cast<const u32x4*>(at + 256 * (i >> 1) + 32 * (i & 1));
}
__device__ __forceinline__ void read_v(const char* at, u32x4 (&v)[2][4]) {
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const char* p = at + ks * kTilePf + 256 * t;
      const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)p));
      const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(p + 2 * kGroup)));
      v[ks][t] = u32x4{a.x, a.y, b.x, b.y};
    }
}

}  // namespace
}  // namespace ekv
