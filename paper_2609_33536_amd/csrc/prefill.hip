// Chunked-prefill attention over a mixed-fidelity paged prefix for gfx950
// (paper §3.2: BASE blocks are read as their high bytes with a zero low
// byte; App. A: a prefill chunk attends its cached prefix and, causally,
// itself).
//
// A workgroup of 4 waves serves one (sequence, KV head, tile of query
// tokens); a wave works on 32 query "columns" -- (token, head-in-group) pairs.
// The work unit is one pair of blocks, 32 keys (the missing second block of
// a lone last one is masked).  On 32x32x16 matrix cores, per unit:
//   S^T (32 keys x 32 columns) = K (32 x 128) . Q^T, 8 products;
//     lane l holds column l % 32 and keys 8(r/4) + 4(l/32) + r%4, r < 16.
//   online softmax over those 16 scores (+ the partner lane l ^ 32);
//   O^T (128 dims x 32 columns) += V^T . P^T, for P's 16-bit head and its
//     16-bit remainder (P keeps ~16 significant bits), 4 dim tiles x 2
//     key steps x 2.  The P operand of key step k is the lane's own scores
//     r = 8k .. 8k+7, so key index 8(l/32) + i of step k stands for key
//     16k + 8(i/4) + 4(l/32) + i%4; the V^T operand follows the same order.
// V^T operands come straight from LDS with the transposing read
// ds_read_b64_tr_b16: within each 16-lane group it hands lane j element j of
// the rows the group's lanes point at (row 4a + j/4, element j%4), so pointing
// lane 4a + b at key a, dims d + 4b .. gives lane j keys a = 0..3 of dim d + j.
// Column c sees keys p < lim(c) = prefix + (its chunk index) + 1.
//
// Every unit lies in LDS as 16-bit words whatever its kind, so one branch-free
// body serves TARGET and BASE blocks and 8-bit pools: TARGET words are loaded
// straight to their place; bytes (BASE, or 8-bit TARGET) and nibbles (8-bit
// BASE) are loaded raw and widened in place, once per workgroup (a wave widens
// the quarter that it loaded).  When every wave fetched and widened the BASE
// operands for itself, a unit cost a wave 182 vector, 110 scalar and 21 branch
// instructions (its 24 products aside); now 147, 59 and 9.
//
// Two kernels:
//   prefill_kernel        4 waves x 32 columns share every unit (pipelined, or
//                         in rounds of 4 units over contexts of at most 8);
//   prefill_split_kernel  4 waves share 32 columns and take every fourth unit
//                         each: small launches, which leave most CUs idle.
#include <cstdlib>
#include <type_traits>

#include "prefill_device.h"
#include "prefill_plan.h"

namespace ekv {
namespace {

constexpr int kPfWaves = 4;

// One wave's 32 query columns of a (sequence, KV head).
template <typename T, int G>
struct Columns : ColumnState<T> {
  // first column col0 of the sequence's chunk; q0, nq: its rows; prefix, len: its keys
  __device__ __forceinline__ Columns(const PrefillArgs& a, int kvh, int q0, int nq, int len, int col0, int lane) {
    const int col = col0 + (lane & 31), h = lane >> 5;
    const int tq = col / G, head = col % G, prefix = len - nq;
    this->ok = tq < nq;
    this->lim = this->ok ? min(len, prefix + tq + 1) : len;
    this->lim_all = min(len, prefix + col0 / G + 1);
    this->row = ((size_t)(q0 + (this->ok ? tq : 0)) * a.num_q_heads + (size_t)kvh * G + head) * kHeadDim;
    this->load_queries(a.q, a.scale_log2, h);
  }
};

// Dim tile t of a column's output: this lane holds dims 32 t + 8 u + 4 h .. + 3.
template <typename T>
__device__ __forceinline__ void store_tile(const PrefillArgs& a, size_t row, const f32x16& o, float inv, int t, int h) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const size_t idx = row + 32 * t + 8 * u + 4 * h;
    store_pair<T>(a.out, idx, o[4 * u] * inv, o[4 * u + 1] * inv, a.out_fp32);
    store_pair<T>(a.out, idx + 2, o[4 * u + 2] * inv, o[4 * u + 3] * inv, a.out_fp32);
  }
}

// A sequence's rows and keys, clamped into q, out and the table.
struct Extent {
  int q0, nq, len;
  __device__ __forceinline__ Extent(const PrefillArgs& a, int s) {
    q0 = min(max(a.cu_q[s], 0), a.total_q);
    nq = min(max(a.cu_q[s + 1], q0), a.total_q) - q0;
    len = max(0, min(a.seq_lens[s], a.max_blocks * kPage));
  }
  // keys that chunk row t sees, at least 1
  __device__ __forceinline__ int seen(int t) const { return max(1, min(len, len - nq + t + 1)); }
};

__device__ __forceinline__ PrefillPlace place(const PrefillArgs& a, int tiles) {
  return place_workgroup(blockIdx.x, blockIdx.y, gridDim.x, gridDim.y, tiles, a.num_kv_heads, a.batch, a.spread != 0);
}

// ---- 4 waves x 32 columns over shared units --------------------------------
// Software pipeline, one barrier a unit: the body of unit i runs the softmax of
// unit i while the matrix cores run the P.V products of unit i - 1 and the
// scores of unit i + 1 (both in the same basic block, so the compiler
// interleaves them), reads K of unit i + 1 and V of unit i, widens unit i + 2
// and issues the loads of unit i + 3.  4 slots, 66,560 B of LDS: two
// workgroups, two waves per SIMD (228-236 registers).
// Measured in one run against the kernel before (32-key units fetched and
// widened per wave, no pipeline), append of the chunk included: 8B chunked
// prefill (16 x (2048 prefix, half BASE, + 512), 32 / 8 heads, bf16) 537 ->
// 481 us; 8-bit pool, 2 x (8192 + 1024), 64 / 8 heads 958 -> 852 us; 3 short
// fp16 prompts 36 -> 28 us.
// What bounds it: matrix work under the power limit.  The kernel runs 1.5x the
// algorithmic flops (P's remainder); with random operands a plain 8192^3 bf16
// product reaches 1.2-1.3 PFLOP/s on this card (1.7 with zeros), which is
// ~370 us for this work, and leaving out the exponentials or the LDS reads
// changes the time by only 2-4 %.  Not kept: 64 columns per wave with one wave
// per SIMD (half the LDS reads, but a lone wave issues a vector instruction
// only every ~4.9 cycles: 4-6 % slower); the remainders p - head by
// v_dot2_f32_bf16 (fewer instructions, but they occupy the matrix pipe: 5 % slower).
constexpr int kPfRing = 4;
// Contexts of at most kPfFew units skip the pipeline, whose fill and drain (the
// loads past the last unit, a unit of products each before the first and after
// the last) cost more there than it hides: the ring is filled with up to 4 units
// at once, and a wave works through them without a barrier.  Measured (us, bf16,
// pipeline / rounds): 64 prompts of up to 16 rows, 16 / 16 heads 12.9 / 10.4, of up
// to 77 rows, 64 / 8 heads 47.8 / 44.7; 5-8 units, 16 x (200 + up to 77), 32 / 8
// heads 20.0 / 18.2, 8-bit, 64 / 8 heads 26.4 / 24.8.
constexpr int kPfFew = 8;

template <typename T, int G, bool ELASTIC, bool F8>
__global__ __launch_bounds__(64 * kPfWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void prefill_kernel(PrefillArgs a) {
  __shared__ __attribute__((aligned(16))) char ring[kPfRing * kSlotPf];
  constexpr int kTileTok = kPfWaves * kPfCols / G;
  const int tiles = (a.max_q_len + kTileTok - 1) / kTileTok;
  const PrefillPlace at = place(a, tiles);
  const int s = at.seq, kvh = at.kv_head, tile = at.tile;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const Extent x(a, s);
  const int t_begin = tile * kTileTok;
  if (t_begin >= x.nq) return;   // uniform over the workgroup

  Columns<T, G> col(a, kvh, x.q0, x.nq, x.len, t_begin * G + wave * kPfCols, lane);
  const int nblk = (x.seen(min(x.nq, t_begin + kTileTok) - 1) + kPage - 1) / kPage;
  PairTable<ELASTIC, F8> table(a, s, kvh, nblk, lane);
  const int units = table.units;
  // the units this wave's own columns see (none if it has no column)
  const int t_wave = t_begin + wave * kPfCols / G;
  const int own_units = t_wave >= x.nq ? 0 : (x.seen(min(x.nq, t_wave + (kPfCols + G - 1) / G) - 1) + 31) >> 5;
  const int valid = min(x.len, nblk * kPage);   // V rows of keys at or past this are zeroed
  const Stager<F8> stager(lane, a.num_kv_heads);
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_ptr)&ring[0]);
  const char* k_at = ring + k_read_offset(lane);
  const char* v_at = ring + v_read_offset(lane);
  auto slot_of = [](int u) -> uint32_t { return (uint32_t)(u & (kPfRing - 1)) * kSlotPf; };

  int issued = 0;
  uint32_t modes = 0;       // bit 0: the unit issued last is BASE
  auto issue = [&]() {      // (past the last unit, its loads again, into a slot that nothing reads)
    const int u = min(issued, units - 1);
    const bool base = table.seek(u, lane);
    stager.load(table.tile(u, wave >> 1), base, wave, lds + slot_of(issued));
    modes = (modes << 1) | (base ? 1u : 0u);
    ++issued;
  };
  // this wave's quarter of unit u, when IN_FLIGHT units after it may still be loading
  auto stage = [&](int u, auto in_flight) {
    wait_loads<Stager<F8>::kLoads * decltype(in_flight)::value>();
    stager.widen(ring + slot_of(u), ELASTIC && ((modes >> (issued - 1 - u)) & 1u) != 0u, wave, 32 * u, valid, lane);
  };

  if (units <= kPfFew) {
#pragma unroll 1
    for (int u0 = 0; u0 < units; u0 += kPfRing) {
      const int u1 = min(units, u0 + kPfRing);
      if (u0 > 0) barrier();   // every wave is done with the ring
#pragma unroll 1
      for (int u = u0; u < u1; ++u) issue();
#pragma unroll 1
      for (int u = u0; u < u1; ++u) stage(u, std::integral_constant<int, 0>{});
      barrier();
#pragma unroll 1
      for (int u = u0; u < min(u1, own_units); ++u) {
        u32x4 k[8], v[2][4], hi[2], lo[2];
        read_k(k_at + slot_of(u), k);
        read_v(v_at + slot_of(u), v);
        f32x16 sc = col.scores(k);
        const float c = col.mask(sc, 32 * u, h);
        float shift;
        if (col.advance(sc, c, &shift)) col.rescale(fast_exp2(shift));
        col.l += col.probabilities(sc, c, col.m, hi, lo);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          col.accumulate(v[ks], hi[ks]);
          col.accumulate(v[ks], lo[ks]);
        }
      }
    }
  } else {
    u32x4 hi[2], lo[2], k[8], v[2][4];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      hi[ks] = lo[ks] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int t = 0; t < 4; ++t) v[ks][t] = u32x4{0u, 0u, 0u, 0u};
    }
    auto products = [&]() {   // O += V^T P^T of the unit whose P and V are in registers
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        col.accumulate(v[ks], hi[ks]);
        col.accumulate(v[ks], lo[ks]);
      }
    };
#pragma unroll 1
    for (int u = 0; u < kPfRing - 1; ++u) issue();
    stage(0, std::integral_constant<int, kPfRing - 2>{});
    stage(1, std::integral_constant<int, kPfRing - 3>{});
    barrier();
    read_k(k_at, k);
    f32x16 sc = col.scores(k);

#pragma unroll 1
    for (int i = 0; i < units; ++i) {
      barrier();   // units i and i + 1 are whole; unit i - 1's slot is free
      issue();
      if (i < own_units) {
        const float c = col.mask(sc, 32 * i, h);
        float shift;
        const bool moved = col.advance(sc, c, &shift);
        read_k(k_at + slot_of(i + 1), k);
        products();
        read_v(v_at + slot_of(i), v);
        const f32x16 next = col.scores(k);
        u32x4 nhi[2], nlo[2];
        float sum = col.probabilities(sc, c, col.m, nhi, nlo);
        // (kept in this block, beside the products: not sunk below the rescale's branch)
        asm volatile("" : "+v"(nhi[0]), "+v"(nhi[1]), "+v"(nlo[0]), "+v"(nlo[1]), "+v"(sum));
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          hi[ks] = nhi[ks];
          lo[ks] = nlo[ks];
        }
        sc = next;
        if (moved) col.rescale(fast_exp2(shift));   // (unit i - 1's products, under the old reference, are in)
        col.l += sum;
      }
      stage(i + 2, std::integral_constant<int, kPfRing - 3>{});
    }
    wait_loads<0>();   // no load may land after the workgroup has ended
    products();
  }

  const float inv = 1.0f / col.total();
  if (col.ok) {
#pragma unroll
    for (int t = 0; t < 4; ++t) store_tile<T>(a, col.row, col.o[t], inv, t, h);
  }
}

// ---- 4 waves share 32 columns and divide the units --------------------------
// A small chunk gives few workgroups of 128 columns, each a serial chain over
// its units (~0.7 us a unit, two LDS round trips, the matrix chain and the
// softmax among them) while most CUs idle.  Here a workgroup has 32 columns and
// wave w takes units w, w + 4, ...: a quarter of the chain, four times the
// workgroups.  A wave loads and widens its units alone (two slots of its own,
// no barrier in the loop); the waves' (o, m, l) are merged through LDS.
// Three fp16 prompts of 17-130 tokens over prefixes of up to 700: 28.8 -> 17.2 us;
// one 4715-token context + 3 rows, 32 / 8 heads: 92 -> 43.
template <typename T, int G, bool ELASTIC, bool F8>
__global__ __launch_bounds__(64 * kPfWaves) __attribute__((amdgpu_waves_per_eu(1, 1))) void prefill_split_kernel(PrefillArgs a) {
  __shared__ __attribute__((aligned(16))) char ring[kPfWaves * 2 * kSlotPf];
  constexpr int kTileTok = kPfCols / G;
  const int tiles = (a.max_q_len + kTileTok - 1) / kTileTok;
  const PrefillPlace at = place(a, tiles);
  const int s = at.seq, kvh = at.kv_head, tile = at.tile;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const Extent x(a, s);
  const int t_begin = tile * kTileTok;
  if (t_begin >= x.nq) return;   // uniform over the workgroup

  Columns<T, G> col(a, kvh, x.q0, x.nq, x.len, t_begin * G, lane);
  const int nblk = (x.seen(min(x.nq, t_begin + kTileTok) - 1) + kPage - 1) / kPage;
  PairTable<ELASTIC, F8> table(a, s, kvh, nblk, lane);
  const int units = table.units;
  const int valid = min(x.len, nblk * kPage);   // V rows of keys at or past this are zeroed
  const Stager<F8> stager(lane, a.num_kv_heads);
  char* own = ring + wave * 2 * kSlotPf;
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_ptr)own);
  const uint32_t k_at = k_read_offset(lane), v_at = v_read_offset(lane);
  constexpr int kUnitLoads = 4 * Stager<F8>::kLoads;

  bool base_of[2] = {false, false};   // the units in slots 0 and 1
  auto issue = [&](int u, int slot) {
    const bool base = table.seek(u, lane);
#pragma unroll
    for (int q = 0; q < 4; ++q) stager.load(table.tile(u, q >> 1), base, q, lds + slot * kSlotPf);
    base_of[slot] = base;
  };
  auto unit = [&](int u, int slot) {
    char* at = own + slot * kSlotPf;
    if (u + kPfWaves < units) wait_loads<kUnitLoads>();
    else wait_loads<0>();
#pragma unroll
    for (int q = 0; q < 4; ++q) stager.widen(at, base_of[slot], q, 32 * u, valid, lane);
    u32x4 k[8], v[2][4], hi[2], lo[2];
    read_k(at + k_at, k);
    read_v(at + v_at, v);
    f32x16 sc = col.scores(k);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot has been read
    if (u + 2 * kPfWaves < units) issue(u + 2 * kPfWaves, slot);
    const float c = col.mask(sc, 32 * u, h);
    float shift;
    // (columns that see none of this wave's keys yet keep the reference -inf)
    if (col.advance(sc, c, &shift)) col.rescale(shift == shift ? fast_exp2(shift) : 1.0f);
    col.l += col.probabilities(sc, c, col.m == -__builtin_inff() ? 0.f : col.m, hi, lo);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      col.accumulate(v[ks], hi[ks]);
      col.accumulate(v[ks], lo[ks]);
    }
  };
  if (wave < units) issue(wave, 0);
  if (wave + kPfWaves < units) issue(wave + kPfWaves, 1);
#pragma unroll 1
  for (int u = wave; u < units; u += 2 * kPfWaves) {
    unit(u, 0);
    if (u + kPfWaves < units) unit(u + kPfWaves, 1);
  }

  // ---- merge: wave w sums dim tile w of the four waves ----
  const float l = col.total();
  barrier();   // every wave is done with the slots (its last loads have been waited for)
  f32x4* parts = reinterpret_cast<f32x4*>(ring);                                  // [wave][tile][4][lane]
  float2* ml = reinterpret_cast<float2*>(ring + kPfWaves * 16 * 64 * sizeof(f32x4));   // [wave][lane]
  ml[64 * wave + lane] = make_float2(col.m, l);
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      parts[((wave * 4 + t) * 4 + r) * 64 + lane] =
          f32x4{col.o[t][4 * r], col.o[t][4 * r + 1], col.o[t][4 * r + 2], col.o[t][4 * r + 3]};
  barrier();
  float2 m[kPfWaves];
  float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
  for (int w = 0; w < kPfWaves; ++w) {
    m[w] = ml[64 * w + lane];
    top = fmaxf(top, m[w].x);
  }
  f32x16 o = f32x16{};
#pragma unroll
  for (int w = 0; w < kPfWaves; ++w) {
    const float f = fast_exp2(m[w].x - top);
    sum += f * m[w].y;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const f32x4 p = parts[((w * 4 + wave) * 4 + r) * 64 + lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[4 * r + e] += f * p[e];
    }
  }
  if (col.ok) store_tile<T>(a, col.row, o, 1.0f / sum, wave, h);
}

template <typename T, int G, bool F8>
hipError_t launch_typed(PrefillArgs a, bool elastic, hipStream_t st) {
  a.spread = spread_tiles((int64_t)a.batch * a.num_kv_heads, a.total_q, (int64_t)a.batch * a.max_q_len);
  constexpr int kSplitTok = kPfCols / G;
  const int64_t split = (int64_t)((a.max_q_len + kSplitTok - 1) / kSplitTok) * a.num_kv_heads * a.batch;
  // (EKV_PREFILL_SPLIT = 0 or 1 overrides, for tests and measurements)
  const char* forced = getenv("EKV_PREFILL_SPLIT");
  if (forced ? atoi(forced) != 0 : divide_units(split, (int64_t)a.max_q_len * G, a.max_len, a.len_stated != 0)) {
    const dim3 grid((unsigned)(split / a.batch), a.batch);
    if (elastic) hipLaunchKernelGGL((prefill_split_kernel<T, G, true, F8>), grid, dim3(64 * kPfWaves), 0, st, a);
    else hipLaunchKernelGGL((prefill_split_kernel<T, G, false, F8>), grid, dim3(64 * kPfWaves), 0, st, a);
    return hipGetLastError();
  }
  constexpr int kTileTok = kPfWaves * kPfCols / G;
  const int tiles = (a.max_q_len + kTileTok - 1) / kTileTok;
  const dim3 grid((unsigned)tiles * a.num_kv_heads, a.batch);
  if (elastic) hipLaunchKernelGGL((prefill_kernel<T, G, true, F8>), grid, dim3(64 * kPfWaves), 0, st, a);
  else hipLaunchKernelGGL((prefill_kernel<T, G, false, F8>), grid, dim3(64 * kPfWaves), 0, st, a);
  return hipGetLastError();
}

template <typename T, bool F8>
hipError_t launch_group(const PrefillArgs& a, int group, bool elastic, hipStream_t st) {
  switch (group) {
    case 1: return launch_typed<T, 1, F8>(a, elastic, st);
    case 2: return launch_typed<T, 2, F8>(a, elastic, st);
    case 4: return launch_typed<T, 4, F8>(a, elastic, st);
    case 8: return launch_typed<T, 8, F8>(a, elastic, st);
    case 16: return launch_typed<T, 16, F8>(a, elastic, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_prefill(const PrefillArgs& a, int dtype, int group, bool elastic, hipStream_t st) {
  if (a.batch == 0 || a.max_q_len == 0) return hipSuccess;
  if (dtype == 3) return launch_group<Fp16, true>(a, group, elastic, st);   // 8-bit pool, FP16 queries
  return dtype == 0 ? launch_group<Bf16, false>(a, group, elastic, st) : launch_group<Fp16, false>(a, group, elastic, st);
}

}  // namespace ekv
