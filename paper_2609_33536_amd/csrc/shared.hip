// Decode attention over shared prefixes for gfx950: sequences in groups, each
// group behind one prefix whose K and V are read once for all of its sequences.
//
// For sequence s of group p and query head h (KV head h / G),
//   out[s][h] = softmax(scale q . [K_prefix(p); K_s]^T) [V_prefix(p); V_s],
// split over keys: a piece is a run of 32-key units of one segment, and leaves
// for each of its query columns the reference max m, the sum l of exp2(s - m)
// and the unnormalised output o.  The pieces of a column, the prefix's and the
// sequence's own, are joined by the merge kernel:
//   out = sum_k 2^(m_k - M) o_k / sum_k 2^(m_k - M) l_k,  M = max_k m_k.
//
// One launch works on three kinds of segments, each kind on workgroups of its own:
//   tile   a prefix with more than 32 query columns (sequence of the group, head of
//          the KV head's G): 4 waves x 32 columns share every unit, pipelined as
//          in prefill.hip; without a causal limit;
//   few    a prefix with at most 32 columns: a wave streams its units alone;
//   own    a sequence's own tokens, G columns: likewise.
// The workgroups are divided between the kinds by the work that each has, a kind's
// units are one flat space, and a workgroup (tile) or wave (few, own) takes an
// equal run of it, crossing segments.  Piece k of a segment is therefore made by
// worker w_first + k, and its slot of partials follows from the segment and the worker.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "prefill_device.h"
#include "shared_plan.h"
#include "wave_scan.h"

namespace ekv {
namespace {

constexpr int kWaves = 4;
constexpr int kRing = 4;

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return min(max(x, lo), hi); }
// The reference of a column all of whose scores so far are -inf: its weights are then 0, not NaN.
__device__ __forceinline__ float finite_or_zero(float m) { return m == -__builtin_inff() ? 0.f : m; }
__device__ __forceinline__ int units_of(int len) { return (len + 2 * kPage - 1) / (2 * kPage); }

// What the prefixes before a chunk of 64 amount to.
struct GroupSums {
  int chunk = 0;                           // the chunk's first prefix
  int start = 0;                           // the group boundary so far
  int tile_units = 0, tile_slots = 0, few_units = 0, few_slots = 0;
};

// 64 prefixes, one a lane: their sequences, units, kind, and where their units
// and slots begin in their kind's.  The group boundaries are clamped into the
// batch and made nondecreasing, so that groups never overlap.
struct Groups {
  int start, count, units, len;
  int tiles, wide;                         // tiles of 128 and groups of 32 columns (tile kind; 0 otherwise)
  bool few;
  int base, slot;                          // of this prefix in its kind's units and slots

  // the chunk at `sums`; advances `sums` past it
  __device__ __forceinline__ Groups(const SharedArgs& a, GroupSums& sums, int lane) {
    const int p = sums.chunk + lane, hkv = a.num_kv_heads;
    const bool in = p < a.prefix.rows;
    const int s0 = in ? clamp_to(a.starts[p], 0, a.own.rows) : 0, s1 = in ? clamp_to(a.starts[p + 1], 0, a.own.rows) : 0;
    len = in ? clamp_to(a.prefix.lens[p], 0, a.prefix.len_cap) : 0;
    start = max(max_scan(s0), sums.start);
    const int end = max(start, s1);
    count = in ? end - start : 0;
    const int columns = count << a.log2_group;
    units = columns > 0 ? units_of(len) : 0;
    few = columns <= kPfCols;
    tiles = units > 0 && !few ? (columns + kWaves * kPfCols - 1) / (kWaves * kPfCols) : 0;
    wide = units > 0 && !few ? (columns + kPfCols - 1) / kPfCols : 0;
    const int u_t = hkv * tiles * units, n_t = hkv * wide;
    const int u_f = few ? hkv * units : 0, n_f = few && units > 0 ? hkv : 0;
    const int iu_t = sum_scan(u_t), in_t = sum_scan(n_t), iu_f = sum_scan(u_f), in_f = sum_scan(n_f);
    base = few ? sums.few_units + iu_f - u_f : sums.tile_units + iu_t - u_t;
    slot = few ? sums.few_slots + in_f - n_f : sums.tile_slots + in_t - n_t;
    sums.chunk += 64;
    sums.tile_units += last_lane(iu_t);
    sums.tile_slots += last_lane(in_t);
    sums.few_units += last_lane(iu_f);
    sums.few_slots += last_lane(in_f);
    sums.start = last_lane(max(max_scan(end), sums.start));
  }
};

// 64 sequences, one a lane: their own tokens and where their units begin.
struct SequenceSums {
  int chunk = 0, units = 0;
};
struct Sequences {
  int len, units, base;
  __device__ __forceinline__ Sequences(const SharedArgs& a, SequenceSums& sums, int lane) {
    const int s = sums.chunk + lane;
    len = s < a.own.rows ? clamp_to(a.own.lens[s], 0, a.own.len_cap) : 0;
    units = units_of(len);
    const int n = a.num_kv_heads * units, incl = sum_scan(n);
    base = sums.units + incl - n;
    sums.chunk += 64;
    sums.units += last_lane(incl);
  }
};

__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// A run of units of one segment, as a worker meets it.
struct Piece {
  int row, kvh, len;         // table row of its part, KV head, tokens of the row
  int u0, u1;                // units
  int seq0, columns;         // the first column's sequence; columns from there
  int slot;                  // where its partials go (wide or own slots)
};

// ---- pieces -----------------------------------------------------------------

template <typename T, bool ELASTIC, bool F8>
struct Worker {
  const SharedArgs& a;
  char* ring;
  int wave, lane, h;
  Stager<F8> stager;

  __device__ __forceinline__ Worker(const SharedArgs& a_, char* ring_)
      : a(a_), ring(ring_), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63),
        h((threadIdx.x & 63) >> 5), stager(threadIdx.x & 63, a_.num_kv_heads) {}

  // the 32 columns from `first` on of a piece: sequence seq0 + column / G, head column % G of the KV head
  __device__ __forceinline__ void columns(ColumnState<T>& col, const Piece& x, int first) const {
    const int c = first + (lane & 31);
    col.ok = c < x.columns;
    col.lim = col.lim_all = x.len;
    const int s = x.seq0 + (col.ok ? c >> a.log2_group : 0);
    const int head = (x.kvh << a.log2_group) + (c & ((1 << a.log2_group) - 1));
    col.row = ((size_t)s * a.num_q_heads + (col.ok ? head : 0)) * kHeadDim;
    col.load_queries(a.q, a.scale_log2, h);
  }

  // partials: 16-byte chunk c (dims 4 c .. + 3) of the slot's `width` columns side by side
  __device__ __forceinline__ void store(const ColumnState<T>& col, float* o, float* ml, int slot, int slots, int width) const {
    const float l = col.total();
    if (!col.ok || (unsigned)slot >= (unsigned)slots) return;
    const int c = lane & 31;
    f32x4* at = reinterpret_cast<f32x4*>(o) + (size_t)slot * 32 * width + c;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        at[(8 * t + 2 * u + h) * width] =
            f32x4{col.o[t][4 * u], col.o[t][4 * u + 1], col.o[t][4 * u + 2], col.o[t][4 * u + 3]};
    if (h == 0) reinterpret_cast<float2*>(ml)[(size_t)slot * width + c] = make_float2(col.m, l);
  }

  // 4 waves x 32 columns over the units of one piece (the pipeline of prefill.hip).
  __device__ __forceinline__ void tile(const Piece& x) {
    ColumnState<T> col;
    columns(col, x, wave * kPfCols);
    const bool active = wave * kPfCols < x.columns;
    PairTable<ELASTIC, F8> table(a.prefix, x.row, x.kvh, (x.len + kPage - 1) / kPage, lane, x.u0);
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_ptr)ring);
    const char* k_at = ring + k_read_offset(lane);
    const char* v_at = ring + v_read_offset(lane);
    const int units = x.u1 - x.u0;
    auto slot_of = [](int u) -> uint32_t { return (uint32_t)(u & (kRing - 1)) * kSlotPf; };
    int issued = 0;
    uint32_t modes = 0;   // bit 0: the unit issued last is BASE
    auto issue = [&]() {  // (past the last unit, its loads again, into a slot that nothing reads)
      const int u = x.u0 + min(issued, units - 1);
      const bool base = table.seek(u, lane);
      stager.load(table.tile(u, wave >> 1), base, wave, lds + slot_of(issued));
      modes = (modes << 1) | (base ? 1u : 0u);
      ++issued;
    };
    auto stage = [&](int u, auto in_flight) {
      wait_loads<Stager<F8>::kLoads * decltype(in_flight)::value>();
      stager.widen(ring + slot_of(u), ELASTIC && ((modes >> (issued - 1 - u)) & 1u) != 0u, wave, 2 * kPage * (x.u0 + u),
                   x.len, lane);
    };
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
    for (int u = 0; u < kRing - 1; ++u) issue();
    stage(0, std::integral_constant<int, kRing - 2>{});
    stage(1, std::integral_constant<int, kRing - 3>{});
    barrier();
    read_k(k_at, k);
    f32x16 sc = col.scores(k);
#pragma unroll 1
    for (int i = 0; i < units; ++i) {
      barrier();   // units i and i + 1 are whole; unit i - 1's slot is free
      issue();
      if (active) {
        const float c = col.mask(sc, 2 * kPage * (x.u0 + i), h);
        float shift;
        const bool moved = col.advance(sc, c, &shift);
        read_k(k_at + slot_of(i + 1), k);
        products();
        read_v(v_at + slot_of(i), v);
        const f32x16 next = col.scores(k);
        u32x4 nhi[2], nlo[2];
        float sum = col.probabilities(sc, c, finite_or_zero(col.m), nhi, nlo);
        // (kept in this block, beside the products: not sunk below the rescale's branch)
        asm volatile("" : "+v"(nhi[0]), "+v"(nhi[1]), "+v"(nlo[0]), "+v"(nlo[1]), "+v"(sum));
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          hi[ks] = nhi[ks];
          lo[ks] = nlo[ks];
        }
        sc = next;
        if (moved) col.rescale(shift == shift ? fast_exp2(shift) : 1.0f);   // (unit i - 1's products, under the old reference, are in)
        col.l += sum;
      }
      stage(i + 2, std::integral_constant<int, kRing - 3>{});
    }
    wait_loads<0>();   // no load may land in a slot of the next piece, or after the workgroup has ended
    products();
    if (active) store(col, a.o_wide, a.ml_wide, x.slot + wave, a.wide_slots, kPfCols);
    barrier();         // every wave is done with the ring
  }

  // One wave's columns over the units of one piece, alone, in the wave's own slot.
  __device__ __forceinline__ void stream(const SharedPart& part, const Piece& x, bool few) {
    ColumnState<T> col;
    columns(col, x, 0);
    PairTable<ELASTIC, F8> table(part, x.row, x.kvh, (x.len + kPage - 1) / kPage, lane, x.u0);
    char* slot = ring + wave * kSlotPf;
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_ptr)slot);
    const uint32_t k_at = k_read_offset(lane), v_at = v_read_offset(lane);
    bool base = false;
    auto issue = [&](int u) {
      base = table.seek(u, lane);
#pragma unroll
      for (int q = 0; q < 4; ++q) stager.load(table.tile(u, q >> 1), base, q, lds);
    };
    issue(x.u0);
#pragma unroll 1
    for (int u = x.u0; u < x.u1; ++u) {
      wait_loads<0>();
#pragma unroll
      for (int q = 0; q < 4; ++q) stager.widen(slot, base, q, 2 * kPage * u, x.len, lane);
      u32x4 k[8], v[2][4], hi[2], lo[2];
      read_k(slot + k_at, k);
      read_v(slot + v_at, v);
      f32x16 sc = col.scores(k);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot has been read
      if (u + 1 < x.u1) issue(u + 1);
      const float c = col.mask(sc, 2 * kPage * u, h);
      float shift;
      if (col.advance(sc, c, &shift)) col.rescale(shift == shift ? fast_exp2(shift) : 1.0f);
      col.l += col.probabilities(sc, c, finite_or_zero(col.m), hi, lo);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        col.accumulate(v[ks], hi[ks]);
        col.accumulate(v[ks], lo[ks]);
      }
    }
    if (few) store(col, a.o_wide, a.ml_wide, x.slot, a.wide_slots, kPfCols);
    else store(col, a.o_own, a.ml_own, x.slot, a.own_slots, 1 << a.log2_group);
  }
};

// ---- the kernel ---------------------------------------------------------------

template <typename T, bool ELASTIC, bool F8>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void shared_kernel(SharedArgs a) {
  __shared__ __attribute__((aligned(16))) char ring[kRing * kSlotPf];
  Worker<T, ELASTIC, F8> worker(a, ring);
  const int lane = worker.lane, hkv = a.num_kv_heads;

  // the work of each kind
  GroupSums g;
#pragma unroll 1
  while (g.chunk < a.prefix.rows) Groups(a, g, lane);
  int own_units = 0;
#pragma unroll 1
  for (int c = 0; c < a.own.rows; c += 512) {   // (8 loads in flight)
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int s = c + 64 * u + lane;
      own_units += units_of(s < a.own.rows ? clamp_to(a.own.lens[s], 0, a.own.len_cap) : 0);
    }
  }
  own_units = hkv * last_lane(sum_scan(own_units));
  const SharedPlan plan = divide_work(g.tile_units, g.few_units, own_units, (int)gridDim.x, a.min_units, F8);
  const int few_slot0 = g.tile_slots + kWaves * plan.tile_workers;

  if (blockIdx.x == 0 && worker.wave == 0) {   // what the merge needs of all this
    if (lane == 0) *reinterpret_cast<int4*>(a.plan) = int4{plan.tile_run, plan.few_run, plan.own_run, few_slot0};
    int4* at = reinterpret_cast<int4*>(a.plan) + 1;
    GroupSums gs;
#pragma unroll 1
    while (gs.chunk < a.prefix.rows) {
      const int p = gs.chunk + lane;
      const Groups x(a, gs, lane);
      if (p < a.prefix.rows) {
        at[2 * p] = int4{x.base, x.slot, x.units, x.start};
        at[2 * p + 1] = int4{x.tiles, x.wide, x.count, 0};
      }
    }
    int2* sat = reinterpret_cast<int2*>(at + 2 * a.prefix.rows);
    SequenceSums ss;
#pragma unroll 1
    while (ss.chunk < a.own.rows) {
      const int s = ss.chunk + lane;
      const Sequences y(a, ss, lane);
      if (s < a.own.rows) sat[s] = int2{y.base, y.units};
    }
  }

  // the prefix of the worker's kind that holds its unit pos (the search goes on where it ended)
  struct {
    int p = -1, start, count, units, len, tiles, wide, base, slot;
  } at;
  GroupSums gs;
  SequenceSums ss;
  auto find_prefix = [&](int pos, bool few) -> bool {
    if (at.p >= 0 && pos < at.base + hkv * (few ? 1 : at.tiles) * at.units) return true;
#pragma unroll 1
    while (gs.chunk < a.prefix.rows) {
      const GroupSums before = gs;
      const Groups x(a, gs, lane);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(x.units > 0 && x.few == few && x.base <= pos &&
                                                       pos < x.base + hkv * (few ? 1 : x.tiles) * x.units);
      if (!hit) continue;
      const int l = __builtin_ctzll(hit);
      at.p = before.chunk + l;
      at.start = lane_value(x.start, l);
      at.count = lane_value(x.count, l);
      at.units = lane_value(x.units, l);
      at.len = lane_value(x.len, l);
      at.tiles = lane_value(x.tiles, l);
      at.wide = lane_value(x.wide, l);
      at.base = lane_value(x.base, l);
      at.slot = lane_value(x.slot, l);
      gs = before;   // (the next prefix may lie in this chunk)
      return true;
    }
    return false;   // (lengths that changed under the launch)
  };
  auto find_sequence = [&](int pos) -> bool {
    if (at.p >= 0 && pos < at.base + hkv * at.units) return true;
#pragma unroll 1
    while (ss.chunk < a.own.rows) {
      const SequenceSums before = ss;
      const Sequences y(a, ss, lane);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(y.base <= pos && pos < y.base + hkv * y.units);
      if (!hit) continue;
      const int l = __builtin_ctzll(hit);
      at.p = before.chunk + l;
      at.len = lane_value(y.len, l);
      at.units = lane_value(y.units, l);
      at.base = lane_value(y.base, l);
      ss = before;
      return true;
    }
    return false;
  };

  const int w = blockIdx.x;
  if (w < plan.tile_workers) {
    int pos = w * plan.tile_run;
    const int end = min(g.tile_units, pos + plan.tile_run);
#pragma unroll 1
    while (pos < end && find_prefix(pos, false)) {
      const int off = pos - at.base, seg = off / at.units, tile = seg % at.tiles;
      const int first = tile * kWaves * kPfCols;
      Piece pc;
      pc.row = at.p;
      pc.kvh = seg / at.tiles;
      pc.len = at.len;
      pc.u0 = off - seg * at.units;
      pc.u1 = min(at.units, pc.u0 + (end - pos));
      pc.seq0 = at.start + (first >> a.log2_group);
      pc.columns = min((at.count << a.log2_group) - first, kWaves * kPfCols);
      pc.slot = at.slot + pc.kvh * at.wide + kWaves * (tile + w);
      worker.tile(pc);
      pos += pc.u1 - pc.u0;
    }
    return;
  }
  // a wave's units: of the prefixes with few columns, or of the sequences
  const bool few = w < plan.tile_workers + plan.few_workers;
  const int ww = (w - plan.tile_workers - (few ? 0 : plan.few_workers)) * kWaves + worker.wave;
  int pos = ww * (few ? plan.few_run : plan.own_run);
  const int end = min(few ? g.few_units : own_units, pos + (few ? plan.few_run : plan.own_run));
#pragma unroll 1
  while (pos < end && (few ? find_prefix(pos, true) : find_sequence(pos))) {
    Piece pc;
    int units, off;
    if (few) {
      pc.row = at.p;
      pc.len = at.len;
      pc.seq0 = at.start;
      pc.columns = at.count << a.log2_group;
      pc.slot = few_slot0 + at.slot;
      units = at.units;
      off = pos - at.base;
    } else {
      pc.row = pc.seq0 = at.p;
      pc.len = at.len;
      pc.columns = 1 << a.log2_group;
      pc.slot = at.p * hkv;
      units = at.units;
      off = pos - at.base;
    }
    pc.kvh = off / units;
    pc.u0 = off - pc.kvh * units;
    pc.u1 = min(units, pc.u0 + (end - pos));
    pc.slot += pc.kvh + ww;
    worker.stream(few ? a.prefix : a.own, pc, few);
    pos += pc.u1 - pc.u0;
  }
}

// ---- merge ---------------------------------------------------------------------
// A workgroup joins 32 columns (32 / G sequences of one KV head): lane l holds
// column l % 32, and wave w the chunks 8 w .. 8 w + 7 (4 each for l / 32).  Pieces
// are taken four at a time, their loads issued together.
template <typename T>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedArgs a) {
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.y, hkv = a.num_kv_heads;
  const int c = blockIdx.x * kPfCols + (lane & 31);
  const int s = c >> a.log2_group, head = c & ((1 << a.log2_group) - 1);
  const bool ok = s < a.own.rows;
  const int4 runs = *reinterpret_cast<const int4*>(a.plan);   // units a worker takes (tile, few, own), slot of the first few worker
  const int4* groups = reinterpret_cast<const int4*>(a.plan) + 1;
  const int2* seqs = reinterpret_cast<const int2*>(groups + 2 * a.prefix.rows);

  // the last prefix that starts at or before this lane's sequence
  int p = -1;
  for (int c0 = 0; c0 < a.prefix.rows; c0 += 64) {
    const int start = c0 + lane < a.prefix.rows ? groups[2 * (c0 + lane)].w : 0x7fffffff;
    const int s_first = (blockIdx.x * kPfCols) >> a.log2_group;
#pragma unroll 1
    for (int k = 0; k < (kPfCols >> a.log2_group); ++k) {
      const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(start <= s_first + k));
      if (s == s_first + k) p += n;
    }
  }
  // pieces: n of them, their first slot and the stride of slots, the columns of a slot and this one's
  int wide_n = 0, wide_slot = 0, wide_step = 1, wide_col = 0, own_n = 0, own_slot = 0;
  if (ok && p >= 0) {
    const int4 g = groups[2 * p], t = groups[2 * p + 1];   // unit base, slot base, units, start; tiles, groups of 32, count
    const int j = ((s - g.w) << a.log2_group) + head;
    if (g.z > 0 && s - g.w < t.z) {
      const bool tile = t.x > 0;
      const int run = tile ? runs.x : runs.y;
      const int off = g.x + (tile ? kvh * t.x + (j >> 7) : kvh) * g.z;
      const int w0 = off / run;
      wide_n = (off + g.z - 1) / run - w0 + 1;
      wide_step = tile ? kWaves : 1;
      wide_slot = tile ? g.y + kvh * t.y + (j >> 5) + kWaves * w0 : runs.w + g.y + kvh + w0;
      wide_col = j & 31;
    }
  }
  if (ok) {
    const int2 y = seqs[s];
    if (y.y > 0) {
      const int off = y.x + kvh * y.y, w0 = off / runs.z;
      own_n = (off + y.y - 1) / runs.z - w0 + 1;
      own_slot = s * hkv + kvh + w0;
    }
  }

  float m = -__builtin_inff(), l = 0.f;
  f32x4 o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto join = [&](const float* os, const float* mls, int n, int slot, int step, int width, int col, int slots) {
    const f32x4* op = reinterpret_cast<const f32x4*>(os);
    const float2* mp = reinterpret_cast<const float2*>(mls);
    constexpr int kAtOnce = 4;
#pragma unroll 1
    for (int k0 = 0; __builtin_amdgcn_ballot_w64(k0 < n); k0 += kAtOnce) {
      float2 ml[kAtOnce];
      f32x4 x[kAtOnce][4];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int at = slot + (k0 + k) * step;
        const bool in = k0 + k < n && (unsigned)at < (unsigned)slots;
        ml[k] = in ? mp[(size_t)at * width + col] : make_float2(-__builtin_inff(), 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x[k][i] = in ? op[(size_t)at * 32 * width + (8 * wave + 2 * i + h) * width + col] : f32x4{0.f, 0.f, 0.f, 0.f};
      }
      float top = m;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, ml[k].x);
      const float base = top == -__builtin_inff() ? 0.f : top;   // (no piece yet: every weight is 0)
      const float f = fast_exp2(m - base);
      l *= f;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= f;
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const float e = fast_exp2(ml[k].x - base);
        l += e * ml[k].y;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += e * x[k][i];
      }
      m = top;
    }
  };
  join(a.o_wide, a.ml_wide, wide_n, wide_slot, wide_step, kPfCols, wide_col, a.wide_slots);
  join(a.o_own, a.ml_own, own_n, own_slot, 1, 1 << a.log2_group, head, a.own_slots);
  if (!ok) return;
  const float inv = wide_n + own_n > 0 ? 1.0f / l : 0.f;   // (a sequence without any token: zeros)
  const size_t row = ((size_t)s * a.num_q_heads + (kvh << a.log2_group) + head) * kHeadDim;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const size_t idx = row + 4 * (8 * wave + 2 * i + h);
    store_pair<T>(a.out, idx, o[i][0] * inv, o[i][1] * inv, a.out_fp32);
    store_pair<T>(a.out, idx + 2, o[i][2] * inv, o[i][3] * inv, a.out_fp32);
  }
}

template <typename T, bool F8>
hipError_t launch_typed(const SharedArgs& a, bool elastic, hipStream_t st) {
  if (elastic) hipLaunchKernelGGL((shared_kernel<T, true, F8>), dim3(a.grid), dim3(64 * kWaves), 0, st, a);
  else hipLaunchKernelGGL((shared_kernel<T, false, F8>), dim3(a.grid), dim3(64 * kWaves), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int columns = a.own.rows << a.log2_group;
  hipLaunchKernelGGL((shared_merge_kernel<T>), dim3((columns + kPfCols - 1) / kPfCols, a.num_kv_heads), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t shared_resident(int* workgroups) {
  static std::atomic<int> cache[64];
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  int cus = cache[dev].load(std::memory_order_relaxed);
  if (cus <= 0) {
    if ((e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev)) != hipSuccess) return e;
    cache[dev].store(cus, std::memory_order_relaxed);
  }
  *workgroups = 2 * cus;   // (66,560 B of LDS and at most 256 registers: two a CU)
  return hipSuccess;
}

hipError_t launch_shared(const SharedArgs& a, int dtype, bool elastic, hipStream_t st) {
  switch (dtype) {
    case 0: return launch_typed<Bf16, false>(a, elastic, st);
    case 1: return launch_typed<Fp16, false>(a, elastic, st);
    case 3: return launch_typed<Fp16, true>(a, elastic, st);   // 8-bit pool, FP16 queries
    default: return hipErrorInvalidValue;
  }
}

}  // namespace ekv
