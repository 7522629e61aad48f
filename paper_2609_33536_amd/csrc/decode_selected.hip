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
// Q follows it, and is chosen so that a wave's loads cover whole 128-byte lines.
#include <algorithm>

#include "attn_device.h"
#include "common.h"
#include "long_context.h"

namespace ekv {
namespace {

constexpr int kTeam = 4;        // waves of a workgroup
constexpr float kLowest = -3.0e38f;   // reference maximum before the first score: finite, so that -inf scores weigh 0

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

// 16-bit pools: lane (n, g) holds for QK step k the 8 elements of chunk
// 2 g + 8 (k / 2) + k % 2 of token n, so that the steps' loads in pairs cover 128 bytes of a
// row, and a BASE row's 16 bytes are two steps.  8-bit pools: chunk 4 g + k (a BASE row's 16 bytes
// are all four).  V: tokens 4 g + i, elements 8 n .. 8 n + 7.
template <bool F8>
__device__ __forceinline__ LaneOffsets lane_offsets(int n, int g) {
  if constexpr (F8)
    return {(uint32_t)(n * kHeadDim + 32 * g), (uint32_t)(4 * g * kHeadDim + 8 * n), (uint32_t)(n * kHeadDim / 2 + 16 * g),
            (uint32_t)(4 * g * kHeadDim / 2 + (4 * n & ~7))};
  else
    return {(uint32_t)(n * 2 * kHeadDim + 32 * g), (uint32_t)(4 * g * 2 * kHeadDim + 16 * n), (uint32_t)(n * kHeadDim + 16 * g),
            (uint32_t)(4 * g * kHeadDim + (8 * n & ~15))};
}

template <typename V>
__device__ __forceinline__ V once(const char* p, uint32_t off) {
  return __builtin_nontemporal_load(reinterpret_cast<const V*>(p + off));
}

// kt, vt: the block's tiles (of its member, for BASE)
template <bool F8, bool ELASTIC>
__device__ __forceinline__ void load_block(Raw<F8>& r, const char* kt, const char* vt, bool base, const LaneOffsets& o) {
  const uint32_t ko = ELASTIC && base ? o.k_base : o.k_target, vo = ELASTIC && base ? o.v_base : o.v_target;
  if constexpr (F8) {
    r.k[0] = once<u32x4>(kt, ko);
    r.k[1] = once<u32x4>(kt, ko + (ELASTIC && base ? 0 : 16));
    const uint32_t row = ELASTIC && base ? kHeadDim / 2 : kHeadDim;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = once<u32x2>(vt, vo + i * row);
  } else {
    const uint32_t odd = ELASTIC && base ? 0 : 16, high = ELASTIC && base ? 64 : 128;
    r.k[0] = once<u32x4>(kt, ko);
    r.k[1] = once<u32x4>(kt, ko + odd);
    r.k[2] = once<u32x4>(kt, ko + high);
    r.k[3] = once<u32x4>(kt, ko + high + odd);
    const uint32_t row = ELASTIC && base ? kHeadDim : 2 * kHeadDim;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = once<u32x4>(vt, vo + i * row);
  }
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
__device__ __forceinline__ void open_block(const Raw<F8>& r, bool base, const u32x4 (&q)[4], int n, f32x4& s, u32x4 (&v)[4]) {
  s = f32x4{0.f, 0.f, 0.f, 0.f};
  if constexpr (F8) {
    if (ELASTIC && base) {
#pragma unroll
      for (int k = 0; k < 4; ++k) s = Mma<T>::qk(nibble_words(r.k[0][k]), q[k], s);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = nibble_words(n & 1 ? r.v[i].y : r.v[i].x);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) s = Mma<T>::qk(byte_words(k & 1 ? r.k[k >> 1].zw : r.k[k >> 1].xy), q[k], s);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = byte_words(r.v[i]);
    }
  } else {
    if (ELASTIC && base) {
#pragma unroll
      for (int k = 0; k < 4; ++k) s = Mma<T>::qk(expand_base8(k & 1 ? r.k[k & 2].zw : r.k[k & 2].xy), q[k], s);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = expand_base8(n & 1 ? r.v[i].zw : r.v[i].xy);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) s = Mma<T>::qk(r.k[k], q[k], s);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = r.v[i];
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

__device__ __forceinline__ void store_agent2(float* p, float a, float b) {
  const uint64_t v = (uint64_t)__float_as_uint(a) | ((uint64_t)__float_as_uint(b) << 32);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_agent2(const float* p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// LDS rows of 132 floats: the rows of 16 heads start 4 banks apart
constexpr int kRow = kHeadDim + 4;
template <int G> struct Joined {
  float o[kTeam][G][kRow];
  float m[kTeam][G], l[kTeam][G];
  int last;
};

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
      phys = (unsigned)block < (unsigned)b.num_blocks ? block : 0;   // never leave the pool
      mode = min(kPage, len - i * kPage) | (i & 1) << 8;
      if constexpr (ELASTIC)
        if (by_tags ? b.tags[at] != 0 : (i >= base_lo && i < base_hi)) mode |= 1 << 9;
    }
  };

  // queries: column c and c + G (or c alone) hold head c; a negative scale negates them (exact)
  const float scale = fabsf(a.scale_log2);
  const uint32_t sign = a.scale_log2 < 0.f ? 0x80008000u : 0u;
  u32x4 q[4];
  const size_t head0 = (size_t)s * a.num_q_heads + (size_t)kvh * G;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int chunk = F8 ? 4 * g + k : 2 * g + 8 * (k >> 1) + (k & 1);
    q[k] = u32x4{0u, 0u, 0u, 0u};
    if (n < (kStack ? 2 * G : G))
      q[k] = *reinterpret_cast<const u32x4*>(a.q + (head0 + n % G) * kHeadDim + 8 * chunk) ^ sign;
  }

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
          open_block<T, F8, ELASTIC>(raw[d][0], m0 & (1 << 9), q, n, sc[0], v[0]);
          open_block<T, F8, ELASTIC>(raw[d][1], m1 & (1 << 9), q, n, sc[1], v[1]);
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
  float* const part_o = a.ws_o + ((size_t)row * a.pieces + piece) * G * kHeadDim;
  float* const part_ml = a.ws_ml + ((size_t)row * a.pieces + piece) * G * 2;
  for (int e = threadIdx.x; e < G * kHeadDim / 2; e += 64 * kTeam) {
    const int h = e / (kHeadDim / 2), d = 2 * (e % (kHeadDim / 2));
    float m = sm.m[0][h];
#pragma unroll
    for (int w = 1; w < kTeam; ++w) m = fmaxf(m, sm.m[w][h]);
    float sum = 0.f, x = 0.f, y = 0.f;
#pragma unroll
    for (int w = 0; w < kTeam; ++w) {
      const float f = fast_exp2(sm.m[w][h] - m);
      sum = fmaf(f, sm.l[w][h], sum);
      x = fmaf(f, sm.o[w][h][d], x);
      y = fmaf(f, sm.o[w][h][d + 1], y);
    }
    if (a.pieces == 1) {
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;   // (no token: zeros)
      store_pair<T>(a.out, (head0 + h) * kHeadDim + d, x * inv, y * inv, a.out_fp32);
    } else {
      store_agent2(part_o + h * kHeadDim + d, x, y);
      if (d == 0) store_agent2(part_ml + 2 * h, m, sum);
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
  const float* const all_o = a.ws_o + (size_t)row * a.pieces * G * kHeadDim;
  const float* const all_ml = a.ws_ml + (size_t)row * a.pieces * G * 2;
  for (int e = threadIdx.x; e < G * kHeadDim / 2; e += 64 * kTeam) {
    const int h = e / (kHeadDim / 2), d = 2 * (e % (kHeadDim / 2));
    float m = kLowest;
    for (int p = 0; p < a.pieces; ++p) m = fmaxf(m, load_agent2(all_ml + 2 * (p * G + h)).x);
    float sum = 0.f, x = 0.f, y = 0.f;
    for (int p = 0; p < a.pieces; ++p) {
      const float2 ml = load_agent2(all_ml + 2 * (p * G + h)), o = load_agent2(all_o + (size_t)(p * G + h) * kHeadDim + d);
      const float f = fast_exp2(ml.x - m);
      sum = fmaf(f, ml.y, sum);
      x = fmaf(f, o.x, x);
      y = fmaf(f, o.y, y);
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    store_pair<T>(a.out, (head0 + h) * kHeadDim + d, x * inv, y * inv, a.out_fp32);
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

int selected_pieces(int64_t rows, int budget) {
  // 512 workgroups fill the chip (two a compute unit); a wave takes at least one step of two blocks
  const int64_t wanted = (512 + rows - 1) / std::max<int64_t>(rows, 1), most = (budget + 2 * kTeam - 1) / (2 * kTeam);
  return (int)std::max<int64_t>(1, std::min(wanted, most));
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
