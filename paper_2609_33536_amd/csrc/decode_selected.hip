// Decode attention over selected blocks, one query token per sequence: for a list of
// logical blocks of each (sequence, KV head),
//   out = softmax(scale q K^T) V   over the tokens of the listed blocks.
//
// A (sequence, KV head)'s list is cut into `pieces` workgroups of 4 waves; a wave takes an
// equal run of the list, two blocks (32 tokens) a step: S^T = K Q^T for the whole query
// group on 16x16x32 MFMA, an online softmax, O^T += V^T P^T (the lane layout of decode.hip,
// with P's 16-bit head and remainder in separate columns for groups of up to 8 heads).
// The waves of a workgroup join their (max, sum, O) in LDS, the pieces through the
// workspace: the last one to arrive adds them up in order.
//
// It is bound by HBM: 8 KiB a block and KV head (4 KiB for an 8-bit pool or a BASE block of a
// 16-bit one), gathered one 4 KiB tile here, one there.  K and V go straight into the registers
// that the products read them from; the head-dim order of the QK product is free, as long as
// Q follows it, and is chosen so that a wave's loads cover whole 128-byte lines.  64 sequences, 8 KV heads, 128 blocks
// each, a quarter of them BASE, 16-bit: 77 us (471 MB, 6.1 TB/s); 48 of 512 blocks, 8-bit, half BASE: 121 us (606 MB, 5.0 TB/s,
// matrix cores 8 %, vector work 35 % of the time); one sequence of 256 blocks 11 us: two dependent reads (list,
// table), two steps of K and V, and the join's three round trips (store, count, load).
#include <algorithm>
#include <type_traits>

#include "attn_device.h"
#include "common.h"
#include "long_context.h"

namespace ekv {
namespace {

constexpr int kTeam = 4;        // waves of a workgroup
constexpr int kMostPieces = 64;
// Reference maximum before the first score: finite, so that scores of -inf weigh 0, and the lowest float, so that no finite
// score lies below it.
constexpr float kLowest = -0x1.fffffep127f;

// One step's K and V as loaded: 16-bit pools 4 + 4 loads of 16 bytes a block, 8-bit ones
// 2 of 16 and 4 of 8.  BASE blocks take the same loads, some of them twice the same address
// or twice as wide as needed (the same lines: the first-level cache has them), so that every
// step has the same number of loads in flight and waits count them exactly.
template <bool F8> struct Raw;
template <> struct Raw<false> {
  u32x4 k[4], v[4];
};
template <> struct Raw<true> {
  u32x4 k[2];
  u32x2 v[4];
};

// A lane's offsets in a (plane, head) tile, TARGET and BASE; see load_block.
struct LaneOffsets {
  uint32_t k_target, v_target, k_base, v_base;
};

// QK step k of lane (n, g) takes 8 elements of token n: of 16-bit pools chunk 4 k + g, so that a load covers 64 bytes of a
// row; of 8-bit ones, where a load of 16 bytes is two steps, chunk 8 (k / 2) + 2 g + k % 2, to the same end.
// V: tokens 4 g + i, elements 8 n .. 8 n + 7.  BASE rows are half as long: a load takes the 16 (8-bit V: 8) bytes that hold
// the lane's half as much.
template <bool F8>
__device__ __forceinline__ constexpr int chunk_of(int g, int k) { return F8 ? 8 * (k >> 1) + 2 * g + (k & 1) : 4 * k + g; }
template <bool F8>
__device__ __forceinline__ LaneOffsets lane_offsets(int n, int g) {
  if constexpr (F8)
    return {(uint32_t)(n * kHeadDim + 16 * g), (uint32_t)(4 * g * kHeadDim + 8 * n), (uint32_t)(n * kHeadDim / 2 + (8 * g & ~15)),
            (uint32_t)(4 * g * kHeadDim / 2 + (4 * n & ~7))};
  else
    return {(uint32_t)(n * 2 * kHeadDim + 16 * g), (uint32_t)(4 * g * 2 * kHeadDim + 16 * n), (uint32_t)(n * kHeadDim + (8 * g & ~15)),
            (uint32_t)(4 * g * kHeadDim + (8 * n & ~15))};
}

// V is read past the caches, K is not: two loads of a wave take the halves of each of K's 128-byte lines, and a
// line read past the first-level cache would come from the second twice.  (64 sequences of 2048 selected tokens, 32 / 8 heads, a quarter
// BASE: 77.5 us; both past the caches 81.6, both through them 84.0.)
template <typename V>
__device__ __forceinline__ V once(const char* p, uint32_t off) {
  return __builtin_nontemporal_load(reinterpret_cast<const V*>(p + off));
}

// kt, vt: the block's tiles (of its member, for BASE)
template <bool F8, bool ELASTIC>
__device__ __forceinline__ void load_block(Raw<F8>& r, const char* kt, const char* vt, bool base, const LaneOffsets& o) {
  const bool half = ELASTIC && base;
  const uint32_t ko = half ? o.k_base : o.k_target, vo = half ? o.v_base : o.v_target;
  constexpr uint32_t kRowBytes = F8 ? kHeadDim : 2 * kHeadDim;
  const uint32_t step = half ? 32 : 64, row = half ? kRowBytes / 2 : kRowBytes;
#pragma unroll
  for (int k = 0; k < (F8 ? 2 : 4); ++k) r.k[k] = *reinterpret_cast<const u32x4*>(kt + (ko + k * step));
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = once<std::remove_reference_t<decltype(r.v[i])>>(vt, vo + i * row);
}

// 8 bytes or 8 nibbles -> the executed FP16 words, in the order of the elements.
__device__ __forceinline__ u32x4 byte_words(u32x2 b) { return expand_base8(b); }
__device__ __forceinline__ u32x4 nibble_words(uint32_t w) {
  const uint32_t even = (w << 4) & 0xF0F0F0F0u, odd = w & 0xF0F0F0F0u;   // byte k: elements 2k, 2k + 1
  return u32x4{perm(odd, even, 0x040C000Cu), perm(odd, even, 0x050C010Cu), perm(odd, even, 0x060C020Cu),
               perm(odd, even, 0x070C030Cu)};
}

// Scores of a block's 16 tokens, and its V rows as 16-bit words.
template <typename T, bool F8, bool ELASTIC>
__device__ __forceinline__ void open_block(const Raw<F8>& r, bool base, const u32x4 (&q)[4], int n, int g, f32x4& s, u32x4 (&v)[4]) {
  s = f32x4{0.f, 0.f, 0.f, 0.f};
  if (ELASTIC && base) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const u32x4 w = r.k[F8 ? k >> 1 : k];
      const u32x2 mine = g & 1 ? w.zw : w.xy;
      if constexpr (F8) s = Mma<T>::qk(nibble_words(k & 1 ? mine.y : mine.x), q[k], s);
      else s = Mma<T>::qk(expand_base8(mine), q[k], s);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (F8) v[i] = nibble_words(n & 1 ? r.v[i].y : r.v[i].x);
      else v[i] = expand_base8(n & 1 ? r.v[i].zw : r.v[i].xy);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (F8) s = Mma<T>::qk(byte_words(k & 1 ? r.k[k >> 1].zw : r.k[k >> 1].xy), q[k], s);
      else s = Mma<T>::qk(r.k[k], q[k], s);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (F8) v[i] = byte_words(r.v[i]);
      else v[i] = r.v[i];
    }
  }
}

// Online softmax over a step's two blocks, of which the first live0 / live1 tokens count, and
// O += V^T P^T; c = |scale| log2(e).  The reference maximum moves only when a step exceeds it by
// more than 2^8 (otherwise P <= 2^8).
template <typename T, int G>
__device__ __forceinline__ void softmax_step(SplitState& st, const f32x4 (&s)[2], u32x4 (&v)[2][4], int live0, int live1,
                                             float c, int g, int n) {
  constexpr bool kStack = 2 * G <= 16;
  float x[2][4];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[b][i] = s[b][i] * c;
  if (min(live0, live1) < kPage) {   // (rows that do not count may hold anything: 0 times NaN would poison the product)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * g + i >= (b ? live1 : live0)) {
          x[b][i] = -__builtin_inff();
          v[b][i] = u32x4{0u, 0u, 0u, 0u};
        }
  }
  float top = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])),
                    fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
  top = head_max(top);
  if (__builtin_amdgcn_ballot_w64(top > st.m + 8.0f)) {
    const float m = fmaxf(st.m, top), alpha = fast_exp2(st.m - m);
    st.l *= alpha;
#pragma unroll
    for (int j = 0; j < 8; ++j) st.o[j] *= alpha;
    st.m = m;
  }
  const float rest = n >= G ? 1.0f : 0.0f;   // (stacked: the columns that hold P's remainder)
  u32x2 head[2], low[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = fast_exp2(x[b][i] - st.m);
    st.l += (p[0] + p[1]) + (p[2] + p[3]);
    if constexpr (kStack) {
      head[b] = u32x2{split_stacked<T>(p[0], p[1], rest), split_stacked<T>(p[2], p[3], rest)};
    } else {
      head[b] = u32x2{split_stacked<T>(p[0], p[1], 0.0f), split_stacked<T>(p[2], p[3], 0.0f)};
      low[b] = u32x2{split_stacked<T>(p[0], p[1], 1.0f), split_stacked<T>(p[2], p[3], 1.0f)};
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const u32x2 a0 = v_operand<false>(v[0], j), a1 = v_operand<false>(v[1], j);
    const u32x4 a = {a0.x, a0.y, a1.x, a1.y};
    st.o[j] = Mma<T>::qk(a, u32x4{head[0].x, head[0].y, head[1].x, head[1].y}, st.o[j]);
    if constexpr (!kStack) st.o[j] = Mma<T>::qk(a, u32x4{low[0].x, low[0].y, low[1].x, low[1].y}, st.o[j]);
  }
}

// Partials pass between workgroups with the agent-scope cache policy (sc1: written through to, and read
// from, the memory side, which every XCD sees), through descriptors of the row's partials.
constexpr int kAgentScope = 16;   // the sc1 bit of the cache-policy operand
__device__ __forceinline__ __amdgpu_buffer_rsrc_t partials(float* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(p, 0, bytes, 0x00020000);
}
__device__ __forceinline__ f32x4 load_agent4(__amdgpu_buffer_rsrc_t r, uint32_t byte) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, byte, 0, kAgentScope));
}
__device__ __forceinline__ float2 load_agent2(__amdgpu_buffer_rsrc_t r, uint32_t byte) {
  return __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(r, byte, 0, kAgentScope));
}

// max / sum over the 16 lanes of a row
template <int N>
__device__ __forceinline__ float ror(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xf, 0xf, true));
}
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, ror<8>(x));
  x = fmaxf(x, ror<4>(x));
  x = fmaxf(x, ror<2>(x));
  return fmaxf(x, ror<1>(x));
}
__device__ __forceinline__ float row_sum(float x) {
  x += ror<8>(x);
  x += ror<4>(x);
  x += ror<2>(x);
  return x + ror<1>(x);
}

// LDS rows of 132 floats: the rows of 16 heads start 4 banks apart
constexpr int kRow = kHeadDim + 4;
template <int G> struct Joined {
  float o[kTeam][G][kRow];
  float m[kTeam][G], l[kTeam][G];
  float weight[kMostPieces][G], inv[G];
  f32x4 part[64 * kTeam];
  int last;
};

template <typename T>
__device__ __forceinline__ void store_chunk(void* out, size_t at, f32x4 x, bool fp32) {
  if (fp32) {
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = x;
  } else {
    float back;
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(out) + at) =
        u32x2{(uint32_t)Mma<T>::round(x[0], &back) | ((uint32_t)Mma<T>::round(x[1], &back) << 16),
              (uint32_t)Mma<T>::round(x[2], &back) | ((uint32_t)Mma<T>::round(x[3], &back) << 16)};
  }
}

template <typename T, int G, bool ELASTIC, bool F8>
__global__ __launch_bounds__(64 * kTeam, 2) void selected_kernel(SelectedArgs a) {
  __shared__ Joined<G> sm;
  constexpr int kDepth = F8 ? 4 : 2;            // steps in flight
  constexpr int kTile = F8 ? kTileBytes / 2 : kTileBytes;
  constexpr bool kStack = 2 * G <= 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const BlockRows& b = a.rows;
  const int hkv = b.num_kv_heads, row = blockIdx.x / (unsigned)a.pieces, piece = blockIdx.x - row * a.pieces;
  const int s = row / (unsigned)hkv, kvh = row - s * hkv;
  const int len = min(max(b.lens[s], 0), b.len_cap), blocks = (len + kPage - 1) / kPage;
  const int listed = a.counts ? min(max(a.counts[row], 0), a.budget) : a.budget;
  // this wave's steps
  const int steps = (listed + 1) / 2, share = (steps + a.pieces * kTeam - 1) / (a.pieces * kTeam);
  const int first = min(steps, (piece * kTeam + wave) * share), last = min(steps, first + share);

  int base_lo = 0, base_hi = 0;
  bool by_tags = false;
  if constexpr (ELASTIC) {
    by_tags = b.tags != nullptr;
    if (b.base) {
      const int p0 = b.base[2 * s], p1 = b.base[2 * s + 1];
      if (p0 >= 0) {
        by_tags = false;
        base_lo = 2 * p0;
        base_hi = 2 * p1;
      }
    }
  }
  // Entries e0 .. e0 + 63 of the list, one a lane: the physical block, and the tokens that
  // count (0 for what is not a block of the sequence) with the mode above them.
  const int entry_end = min(2 * last, listed);
  const int32_t* list = a.selected + (size_t)row * a.budget;
  auto fetch = [&](int e0, int& phys, int& mode) {
    const int e = e0 + lane;
    const int i = e < entry_end ? list[e] : -1;
    phys = mode = 0;
    if ((unsigned)i < (unsigned)blocks) {
      const size_t at = (size_t)s * b.max_blocks + i;
      const int block = b.bt[at];
      const uint8_t tag = (by_tags ? b.tags : reinterpret_cast<const uint8_t*>(b.bt))[at];   // (one round trip)
      phys = (unsigned)block < (unsigned)b.num_blocks ? block : 0;   // never leave the pool
      mode = min(kPage, len - i * kPage) | (i & 1) << 8;
      if constexpr (ELASTIC)
        if (by_tags ? tag != 0 : (i >= base_lo && i < base_hi)) mode |= 1 << 9;
    }
  };

  // queries: column c and c + G (or c alone) hold head c; a negative scale negates them (exact)
  const float scale = fabsf(a.scale_log2);
  const uint32_t sign = a.scale_log2 < 0.f ? 0x80008000u : 0u;
  u32x4 q[4];
  const size_t head0 = (size_t)s * a.num_q_heads + (size_t)kvh * G;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    q[k] = *reinterpret_cast<const u32x4*>(a.q + (head0 + n % G) * kHeadDim + 8 * chunk_of<F8>(g, k));

  SplitState st;
#pragma unroll
  for (int j = 0; j < 8; ++j) st.o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  st.m = kLowest;
  st.l = 0.f;

  const LaneOffsets off = lane_offsets<F8>(n, g);
  const char* const k_plane = reinterpret_cast<const char*>(b.pool) + (size_t)kvh * kTile;
  const size_t block_bytes = (size_t)2 * hkv * kTile, v_plane = (size_t)hkv * kTile;

  // Windows of 64 entries (32 steps); a window's entries are fetched while the one before is worked on.
  int phys, mode, phys_next = 0, mode_next = 0;
  fetch(2 * first, phys, mode);
  const bool used = n < (kStack ? 2 * G : G);   // (the queries' loads are on their way beside the list's)
#pragma unroll
  for (int k = 0; k < 4; ++k) q[k] = used ? q[k] ^ sign : u32x4{0u, 0u, 0u, 0u};
  for (int w0 = first; w0 < last; w0 += 32) {
    fetch(2 * (w0 + 32), phys_next, mode_next);
    const int here = min(32, last - w0);
    Raw<F8> raw[kDepth][2];
    auto load = [&](Raw<F8> (&r)[2], int t) {   // (past the window: its last step again, from the caches)
      t = min(t, here - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int m = __builtin_amdgcn_readlane(mode, 2 * t + h);
        const bool base = m & (1 << 9);
        const char* src = k_plane + (size_t)(unsigned)__builtin_amdgcn_readlane(phys, 2 * t + h) * block_bytes;
        if (ELASTIC && base && (m & (1 << 8))) src += kTile / 2;   // the pair's second member
        load_block<F8, ELASTIC>(r[h], src, src + v_plane, base, off);
      }
    };
#pragma unroll
    for (int d = 0; d < kDepth; ++d) load(raw[d], d);
#pragma unroll 1
    for (int t = 0; t < here; t += kDepth) {
#pragma unroll
      for (int d = 0; d < kDepth; ++d) {
        const int m0 = __builtin_amdgcn_readlane(mode, 2 * min(t + d, here - 1)),
                  m1 = __builtin_amdgcn_readlane(mode, 2 * min(t + d, here - 1) + 1);
        if (t + d < here && ((m0 | m1) & 255)) {
          f32x4 sc[2];
          u32x4 v[2][4];
          open_block<T, F8, ELASTIC>(raw[d][0], m0 & (1 << 9), q, n, g, sc[0], v[0]);
          open_block<T, F8, ELASTIC>(raw[d][1], m1 & (1 << 9), q, n, g, sc[1], v[1]);
          softmax_step<T, G>(st, sc, v, m0 & 255, m1 & 255, scale, g, n);
        }
        load(raw[d], t + d + kDepth);
      }
    }
    phys = phys_next;
    mode = mode_next;
  }

  // ---- the workgroup's waves joined ---------------------------------------
  if constexpr (kStack) stacked_sum<G>(st);
  const float l = head_sum(st.l);
  if (n < G) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* dst = &sm.o[wave][n][32 * g + 8 * r];
      *reinterpret_cast<f32x4*>(dst) = f32x4{st.o[0][r], st.o[1][r], st.o[2][r], st.o[3][r]};
      *reinterpret_cast<f32x4*>(dst + 4) = f32x4{st.o[4][r], st.o[5][r], st.o[6][r], st.o[7][r]};
    }
    if (g == 0) {
      sm.m[wave][n] = st.m;
      sm.l[wave][n] = l;
    }
  }
  __syncthreads();
  constexpr int kChunks = G * kHeadDim / 4, kAll = 64 * kTeam;   // 16-byte chunks of the group's output
  constexpr uint32_t kSlot = G * kHeadDim * sizeof(float), kSlotMl = G * 2 * sizeof(float);
  const auto part_o = partials(a.ws_o + (size_t)row * a.pieces * G * kHeadDim, a.pieces * kSlot);
  const auto part_ml = partials(a.ws_ml + (size_t)row * a.pieces * G * 2, a.pieces * kSlotMl);
#pragma unroll
  for (int c = 0; c < (kChunks + kAll - 1) / kAll; ++c) {
    const int e = c * kAll + (int)threadIdx.x, h = e / (kHeadDim / 4), d = 4 * (e % (kHeadDim / 4));
    if (kChunks < kAll && e >= kChunks) break;
    float m = sm.m[0][h];
#pragma unroll
    for (int w = 1; w < kTeam; ++w) m = fmaxf(m, sm.m[w][h]);
    float sum = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kTeam; ++w) {
      const float f = fast_exp2(sm.m[w][h] - m);
      sum = fmaf(f, sm.l[w][h], sum);
      x += f * *reinterpret_cast<const f32x4*>(&sm.o[w][h][d]);
    }
    if (a.pieces == 1) {
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;   // (no token: zeros)
      store_chunk<T>(a.out, (head0 + h) * kHeadDim + d, x * inv, a.out_fp32);
    } else {
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), part_o, piece * kSlot + 16 * e, 0, kAgentScope);
      if (d == 0)
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, make_float2(m, sum)), part_ml, piece * kSlotMl + 8 * h, 0,
                                              kAgentScope);
    }
  }
  if (a.pieces == 1) return;

  // ---- the pieces joined by the last one ------------------------------------
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's partials have landed
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t before = __hip_atomic_fetch_add(a.counters + row, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sm.last = before == (uint32_t)a.pieces - 1;
    if (sm.last) __hip_atomic_store(a.counters + row, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!sm.last) return;
  asm volatile("" ::: "memory");
  // Thread e holds chunk e (groups of 16 heads: and e + 256) of the pieces r, r + kShares, ..; the
  // first of them are on their way while the weights are worked out.  Past the last piece: beyond the descriptor's
  // bound, which reads zeros and no memory.
  constexpr int kShares = kChunks < kAll ? kAll / kChunks : 1, kHeld = kChunks > kAll ? kChunks / kAll : 1, kAhead = 16 / kHeld;
  const int e = threadIdx.x % kChunks, r = threadIdx.x / kChunks;
  f32x4 v[kAhead][kHeld];
  auto load = [&](int k0) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int p = r + (k0 + u) * kShares;
#pragma unroll
      for (int c = 0; c < kHeld; ++c) v[u][c] = load_agent4(part_o, p < a.pieces ? p * kSlot + 16 * (e + c * kAll) : 0x80000000u);
    }
  };
  load(0);
  if (threadIdx.x < 16 * G) {   // 16 lanes a head, 4 pieces a lane
    const int h = threadIdx.x / 16, j = threadIdx.x % 16;
    float2 ml[kMostPieces / 16];
#pragma unroll
    for (int u = 0; u < kMostPieces / 16; ++u)
      ml[u] = j + 16 * u < a.pieces ? load_agent2(part_ml, (j + 16 * u) * kSlotMl + 8 * h) : make_float2(kLowest, 0.f);
    float m = ml[0].x;
#pragma unroll
    for (int u = 1; u < kMostPieces / 16; ++u) m = fmaxf(m, ml[u].x);
    m = row_max(m);
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < kMostPieces / 16; ++u) {
      const float f = fast_exp2(ml[u].x - m);
      sum = fmaf(f, ml[u].y, sum);
      sm.weight[j + 16 * u][h] = f;
    }
    sum = row_sum(sum);
    if (j == 0) sm.inv[h] = sum == 0.f ? 0.f : 1.0f / sum;
  }
  __syncthreads();
  f32x4 x[kHeld];
#pragma unroll
  for (int c = 0; c < kHeld; ++c) x[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int k0 = 0; r + k0 * kShares < a.pieces; k0 += kAhead) {
    if (k0 > 0) load(k0);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int p = r + (k0 + u) * kShares;
      if (p < a.pieces)
#pragma unroll
        for (int c = 0; c < kHeld; ++c) x[c] += sm.weight[p][(e + c * kAll) / (kHeadDim / 4)] * v[u][c];
    }
  }
  if constexpr (kShares > 1) {
    sm.part[threadIdx.x] = x[0];
    __syncthreads();
    if (r > 0) return;
#pragma unroll
    for (int k = 1; k < kShares; ++k) x[0] += sm.part[e + k * kChunks];
  }
#pragma unroll
  for (int c = 0; c < kHeld; ++c) {
    const int at = e + c * kAll, h = at / (kHeadDim / 4);
    store_chunk<T>(a.out, (head0 + h) * kHeadDim + 4 * (at % (kHeadDim / 4)), x[c] * sm.inv[h], a.out_fp32);
  }
}

template <typename T, int G, bool F8>
hipError_t run_elastic(const SelectedArgs& a, bool elastic, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.rows.batch * a.rows.num_kv_heads * a.pieces)), block(64 * kTeam);
  if (elastic) hipLaunchKernelGGL((selected_kernel<T, G, true, F8>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((selected_kernel<T, G, false, F8>), grid, block, 0, st, a);
  return hipGetLastError();
}

template <typename T, bool F8>
hipError_t run_group(const SelectedArgs& a, int group, bool elastic, hipStream_t st) {
  switch (group) {
    case 1: return run_elastic<T, 1, F8>(a, elastic, st);
    case 2: return run_elastic<T, 2, F8>(a, elastic, st);
    case 4: return run_elastic<T, 4, F8>(a, elastic, st);
    case 8: return run_elastic<T, 8, F8>(a, elastic, st);
    case 16: return run_elastic<T, 16, F8>(a, elastic, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

// A list is cut while its pieces stay within one workgroup a compute unit, where a piece has about 16 blocks
// (a wave two steps) or more: a compute unit's four waves with two steps ahead nearly reach their share of the bandwidth,
// and what a second workgroup there gains the join costs.  Measured in us, pieces up to 256 | up to 512 workgroups in all,
// lists of 256 blocks half BASE, 8 KV heads: 16-bit 4 sequences 16.0 | 18.8, 8 22.4 | 32.7, 15 35.8 | 45.3;
// 8-bit 8 sequences 17.5 | 33.7, 15 24.2 | 34.7.  (8 lists of 256 blocks in 4, 8, 16, 32 pieces: 17.1, 12.6, 10.9, 10.8.)
// 129 to 255 lists are not cut, though some compute units have none then: uncut | in two | in three pieces, 16-bit 17 sequences
// 47.2 | 57.7 | 48.0, 20 49.3 | 60.2 | 50.4, 24 53.1 | 63.7 | 67.9, 31 65.6 | 70.1 | 74.7; 8-bit 17 32.8 | 36.4 | 30.7,
// 24 33.5 | 38.2 | 42.8, 31 35.5 | 41.7 | 50.4.  (16 sequences, in two pieces, 37.6 and 24.1.)
// Lists of up to 32 blocks take less uncut (9.1, in two pieces 9.6).  A little above 256 lists some compute units
// have two workgroups and most one: lists of 128 blocks or more are halved up to 384 of them (33 sequences
// 103.6 -> 87.4, 8-bit 56.5 -> 53.3; 48: 109.6 -> 102.7, 62.6 -> 60.7; but 56: 114.9 -> 124.8, 67.2 -> 76.2).
int selected_pieces(int64_t rows, int blocks) {
  constexpr int kUnits = 256;
  if (blocks <= 32 || rows <= 0) return 1;
  if (rows > kUnits) return rows <= kUnits * 3 / 2 && blocks >= 128 ? 2 : 1;
  return (int)std::min<int64_t>({kUnits / rows, (blocks + 4 * kTeam - 1) / (4 * kTeam), kMostPieces});
}

hipError_t launch_selected(const SelectedArgs& a, int dtype, int group, bool elastic, hipStream_t st) {
  if (a.rows.batch == 0) return hipSuccess;
  switch (dtype) {
    case 0: return run_group<Bf16, false>(a, group, elastic, st);
    case 1: return run_group<Fp16, false>(a, group, elastic, st);
    case 3: return run_group<Fp16, true>(a, group, elastic, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace ekv
