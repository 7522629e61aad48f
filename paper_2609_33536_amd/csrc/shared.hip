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
// One launch works on four kinds of segments (a segment: one KV head of a prefix, or of
// a sequence's own tokens), each kind on workgroups of its own:
//   team   a prefix with more than 128 query columns (sequence of the group, head of the
//          KV head's G): a team of workgroups, one for each tile of 128 columns, takes a
//          run of the prefix's units, so that all of the team read the same K and V at
//          the same time, on one XCD;
//   single a prefix with 33 to 128 columns: one workgroup takes a run of units;
//   few    a prefix with at most 32 columns: a wave streams its units alone;
//   own    a sequence's own tokens, G columns: likewise.
// In a tile of 128, 4 waves x 32 columns share every unit, pipelined as in prefill.hip.
// The workgroups are divided between the kinds by the work that each has.  A kind's
// units are one flat space (for teams, each prefix's are), a worker takes an equal run
// of it and crosses segments.  Piece k of a segment is therefore made by worker
// w_first + k, and its slot of partials follows from the segment and the worker.
#include <algorithm>
#include <atomic>

#include "prefill_device.h"
#include "shared_plan.h"
#include "wave_scan.h"

namespace ekv {
namespace {

constexpr int kWaves = 4;
constexpr int kTileCols = kWaves * kPfCols;
// LDS: 4 slots of K planes and 5 of V planes of a unit (tiles), or a unit's slot per wave (few, own).
constexpr int kVSlots = 5;
constexpr int kVRing = 4 * kPlanePf;
constexpr int kLdsBytes = kVRing + kVSlots * kPlanePf;
static_assert(kLdsBytes >= kWaves * kSlotPf, "a slot for every wave");

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return min(max(x, lo), hi); }
// The reference of a column all of whose scores so far are -inf: its weights are then 0, not NaN.
__device__ __forceinline__ float finite_or_zero(float m) { return m == -__builtin_inff() ? 0.f : m; }
__device__ __forceinline__ int units_of(int len) { return (len + 2 * kPage - 1) / (2 * kPage); }

enum Kind { kNone, kFew, kSingle, kTeam };

// What the prefixes before a chunk of 64 amount to.
struct GroupSums {
  int chunk = 0;                           // the chunk's first prefix
  int start = 0;                           // the group boundary so far
  int few_units = 0, few_segments = 0;     // (a few segment has one slot, besides one a worker)
  int single_units = 0, single_segments = 0, single_slots = 0;
  int team_units = 0, team_tiles = 0, team_slots = 0, team_workers = 0;
};

// 64 prefixes, one a lane: their sequences, units, kind, and where their work and
// slots begin in their kind's.  The group boundaries are clamped into the batch and
// made nondecreasing, so that groups never overlap.
struct Groups {
  int start, count, units, len, kind;
  int tiles, wide;                         // tiles of 128 and groups of 32 columns
  int base, slot;                          // few, single: first unit; team: first worker; first slot
  int run;                                 // team: units of the prefix (all KV heads) that a team takes

  // the chunk at `sums`, with teams of about team_run units; advances `sums` past it
  __device__ __forceinline__ Groups(const SharedArgs& a, GroupSums& sums, int team_run, int lane) {
    const int p = sums.chunk + lane, hkv = a.num_kv_heads;
    const bool in = p < a.prefix.rows;
    const int s0 = in ? clamp_to(a.starts[p], 0, a.own.rows) : 0, s1 = in ? clamp_to(a.starts[p + 1], 0, a.own.rows) : 0;
    len = in ? clamp_to(a.prefix.lens[p], 0, a.prefix.len_cap) : 0;
    start = max(max_scan(s0), sums.start);
    const int end = max(start, s1);
    count = in ? end - start : 0;
    const int columns = count << a.log2_group;
    units = columns > 0 ? units_of(len) : 0;
    tiles = (columns + kTileCols - 1) / kTileCols;
    wide = (columns + kPfCols - 1) / kPfCols;
    kind = units == 0 ? kNone : (columns <= kPfCols ? kFew : (tiles == 1 ? kSingle : kTeam));
    const int all = hkv * units;
    const int teams = kind == kTeam ? (all + team_run - 1) / team_run : 1;
    run = (all + teams - 1) / teams;
    const int few = kind == kFew ? all : 0, single = kind == kSingle ? all : 0, workers = kind == kTeam ? teams * tiles : 0;
    const int single_slot = kind == kSingle ? hkv * wide : 0, team_slot = kind == kTeam ? (hkv + teams) * wide : 0;
    const int if_u = sum_scan(few), if_s = sum_scan(kind == kFew ? hkv : 0), is_u = sum_scan(single), is_s = sum_scan(single_slot);
    const int it_w = sum_scan(workers), it_s = sum_scan(team_slot);
    base = kind == kFew ? sums.few_units + if_u - few
                        : (kind == kSingle ? sums.single_units + is_u - single : sums.team_workers + it_w - workers);
    slot = kind == kFew ? sums.few_segments + if_s - hkv
                        : (kind == kSingle ? sums.single_slots + is_s - single_slot : sums.team_slots + it_s - team_slot);
    sums.chunk += 64;
    sums.few_units += last_lane(if_u);
    sums.few_segments += last_lane(if_s);
    sums.single_units += last_lane(is_u);
    sums.single_segments += hkv * __builtin_popcountll(__builtin_amdgcn_ballot_w64(kind == kSingle));
    sums.single_slots += last_lane(is_s);
    sums.team_units += last_lane(sum_scan(kind == kTeam ? all * tiles : 0));
    sums.team_tiles += last_lane(sum_scan(kind == kTeam ? tiles : 0));
    sums.team_workers += last_lane(it_w);
    sums.team_slots += last_lane(it_s);
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

// The block table of one piece of at most 64 units, a unit a lane: K tile addresses
// of both blocks and the modes, as in PairTable, with the entries of the piece after
// it on their way.
template <bool ELASTIC, bool F8>
struct UnitTable {
  uint64_t pool, block_bytes;
  int num_blocks;
  uint64_t addr0 = 0, addr1 = 0, base_mask = 0;
  int next0 = 0, next1 = 0;
  bool next_base = false;

  __device__ __forceinline__ explicit UnitTable(const SharedPart& part)
      : pool(reinterpret_cast<uint64_t>(part.pool)), block_bytes((uint64_t)2 * part.num_kv_heads * Stager<F8>::kTileP),
        num_blocks(part.num_blocks) {}
  __device__ __forceinline__ void fetch(const SharedPart& part, const Piece& x, int lane) {
    const int u = x.u0 + lane, nblk = (x.len + kPage - 1) / kPage;
    const size_t row = (size_t)x.row * part.max_blocks;
    next0 = next1 = 0;
    next_base = false;
    if (u < x.u1) {
      next0 = part.bt[row + 2 * u];
      next1 = 2 * u + 1 < nblk ? part.bt[row + 2 * u + 1] : next0;   // a lone last block stands in for the missing one (masked)
      if constexpr (ELASTIC) {
        const int b0 = part.bounds ? part.bounds[2 * x.row] : -1;
        if (b0 >= 0) next_base = u >= b0 && u < part.bounds[2 * x.row + 1];
        else if (part.tags) next_base = part.tags[row + 2 * u] != 0;
      }
    }
  }
  __device__ __forceinline__ void enter(int lane, const Piece& x) {
    const int b0 = (unsigned)next0 < (unsigned)num_blocks ? next0 : 0;   // never leave the pool
    const int b1 = (unsigned)next1 < (unsigned)num_blocks ? next1 : 0;
    const uint64_t head = pool + (uint64_t)x.kvh * Stager<F8>::kTileP;
    addr0 = head + (uint64_t)(uint32_t)b0 * block_bytes;
    addr1 = next_base ? addr0 : head + (uint64_t)(uint32_t)b1 * block_bytes;   // (a BASE pair lies in its first block)
    base_mask = __builtin_amdgcn_ballot_w64(next_base);
  }
  __device__ __forceinline__ bool is_base(int i) const { return ELASTIC && ((base_mask >> i) & 1) != 0; }
  __device__ __forceinline__ uint64_t tile(int i, int member) const {
    const uint64_t a = member ? addr1 : addr0;
    uint64_t at = ((uint64_t)(uint32_t)lane_value((int)(a >> 32), i) << 32) | (uint32_t)lane_value((int)a, i);
    asm("s_nop 2" : "+s"(at));   // (3 of the 5 wait states before dma16's load reads it: see PairTable::tile)
    return at;
  }
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
  __device__ __forceinline__ void place(ColumnState<T>& col, const Piece& x, int first) const {
    const int c = first + (lane & 31);
    col.ok = c < x.columns;
    col.lim = col.lim_all = x.len;
    const int s = x.seq0 + (col.ok ? c >> a.log2_group : 0);
    const int head = (x.kvh << a.log2_group) + (c & ((1 << a.log2_group) - 1));
    col.row = ((size_t)s * a.num_q_heads + (col.ok ? head : 0)) * kHeadDim;
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

  // 4 waves x 32 columns over the units of one piece: the pipeline of prefill.hip
  // (softmax of unit i beside the products of unit i - 1 and the scores of unit
  // i + 1, one barrier a unit), but K and V in rings of their own.  K of unit i is
  // read in body i - 1 and V in body i, so 4 K and 5 V slots hold four units ahead:
  // body i issues unit i + 4, waits for K of i + 2 and V of i + 1, and a load has
  // three to four bodies to land where the common ring of 4 left two.  (A prefix's
  // units come from HBM, not from an L2 that sixteen query tiles have warmed.)
  __device__ __forceinline__ void tile(const Piece& x) {
    ColumnState<T> col;
    place(col, x, wave * kPfCols);
    col.load_queries(a.q, a.scale_log2, h);
    const bool active = wave * kPfCols < x.columns;
    PairTable<ELASTIC, F8> table(a.prefix, x.row, x.kvh, (x.len + kPage - 1) / kPage, lane, x.u0);
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_ptr)ring);
    const char* k_at = ring + k_read_offset(lane);
    const char* v_at = ring + kVRing - kPlanePf + v_read_offset(lane);   // (v_read_offset counts from a unit's K)
    const int units = x.u1 - x.u0;
    auto k_slot = [](int u) -> uint32_t { return (uint32_t)(u & 3) * kPlanePf; };
    int issued = 0, v_issue = 0, v_read = 0, v_stage = 0;   // V slots (offsets) of the units at hand
    auto next_v = [](int& at) {
      const int was = at;
      at = at + kPlanePf == kVSlots * kPlanePf ? 0 : at + kPlanePf;
      return was;
    };
    uint32_t modes = 0;   // bit 0: the unit issued last is BASE
    auto issue = [&]() {  // (past the last unit, its loads again, into slots that nothing reads)
      const int u = x.u0 + min(issued, units - 1);
      const bool base = table.seek(u, lane);
      stager.load_planes(table.tile(u, wave >> 1), base, wave, lds + k_slot(issued), lds + kVRing + next_v(v_issue));
      modes = (modes << 1) | (base ? 1u : 0u);
      ++issued;
    };
    auto is_base = [&](int u) { return ELASTIC && ((modes >> (issued - 1 - u)) & 1u) != 0u; };
    auto stage_k = [&](int u) { stager.widen_plane(ring + k_slot(u), is_base(u), wave, lane); };
    auto stage_v = [&](int u) {
      char* at = ring + kVRing + next_v(v_stage);
      stager.widen_plane(at, is_base(u), wave, lane);
      stager.clear_tail(at, wave, 2 * kPage * (x.u0 + u), x.len);
    };
    // everything but the last 5 planes issued (V of unit i + 2, K and V of i + 3 and i + 4) has landed
    auto landed = [&]() { wait_loads<5 * Stager<F8>::kLoads / 2>(); };
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
    for (int u = 0; u < 4; ++u) issue();
    landed();
    stage_k(0);
    stage_k(1);
    stage_v(0);
    barrier();
    read_k(k_at, k);
    f32x16 sc = col.scores(k);
#pragma unroll 1
    for (int i = 0; i < units; ++i) {
      barrier();   // K of unit i + 1 and V of unit i are whole; the slots of K i and V i - 1 are free
      issue();
      const int v_now = next_v(v_read);
      if (active) {
        const float c = col.mask(sc, 2 * kPage * (x.u0 + i), h);
        float shift;
        const bool moved = col.advance(sc, c, &shift);
        read_k(k_at + k_slot(i + 1), k);
        products();
        read_v(v_at + v_now, v);
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
      landed();
      stage_k(i + 2);
      stage_v(i + 1);
    }
    wait_loads<0>();   // no load may land in a slot of the next piece, or after the workgroup has ended
    products();
    if (active) store(col, a.o_wide, a.ml_wide, x.slot + wave, a.wide_slots, kPfCols);
    barrier();         // every wave is done with the rings
  }

  // One wave's columns over a run of units, alone, in the wave's own slot of LDS.
  // `next` gives the run's pieces one after the other, at most 64 units each, and
  // is asked one piece ahead: the block table of a piece is read while the one before
  // is worked on, its first unit is loaded and its queries read when the last unit
  // before has left the slot and the query registers, so that the wave's stream of
  // loads does not stop between segments.
  template <typename Next>
  __device__ __forceinline__ void stream(const SharedPart& part, Next next, float* o, float* ml, int slots, int width) {
    ColumnState<T> col;
    char* slot = ring + wave * kSlotPf;
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_ptr)slot);
    const uint32_t k_at = k_read_offset(lane), v_at = v_read_offset(lane);
    UnitTable<ELASTIC, F8> table(part);
    Piece x, y;               // the piece of the unit at hand, and the one after it
    bool more = next(x);
    if (!more) return;
    table.fetch(part, x, lane);
    table.enter(lane, x);
    bool base = false;
    auto issue = [&](int i) {   // unit i of the table's piece
      base = table.is_base(i);
#pragma unroll
      for (int q = 0; q < 4; ++q) stager.load(table.tile(i, q >> 1), base, q, lds);
    };
    place(col, x, 0);
    issue(0);
    col.load_queries(a.q, a.scale_log2, h);
    more = next(y);
    if (more) table.fetch(part, y, lane);
    int i = 0;                // unit of the piece
#pragma unroll 1
    while (true) {
      const int key0 = 2 * kPage * (x.u0 + i);
      wait_loads<0>();
#pragma unroll
      for (int q = 0; q < 4; ++q) stager.widen(slot, base, q, key0, x.len, lane);
      u32x4 k[8], v[2][4], hi[2], lo[2];
      read_k(slot + k_at, k);
      read_v(slot + v_at, v);
      f32x16 sc = col.scores(k);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot has been read
      const bool last = x.u0 + ++i == x.u1;   // the piece's last unit
      const float c = col.mask(sc, key0, h);
      if (!last) {
        issue(i);
      } else if (more) {
        table.enter(lane, y);
        issue(0);
      }
      float shift;
      if (col.advance(sc, c, &shift)) col.rescale(shift == shift ? fast_exp2(shift) : 1.0f);
      col.l += col.probabilities(sc, c, finite_or_zero(col.m), hi, lo);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        col.accumulate(v[ks], hi[ks]);
        col.accumulate(v[ks], lo[ks]);
      }
      if (!last) continue;
      const bool ends = !more || y.u0 != x.u1 || y.row != x.row || y.kvh != x.kvh;   // (a long segment goes on in the next piece)
      if (ends) store(col, o, ml, x.slot, slots, width);
      if (!more) return;
      if (ends) {
        place(col, y, 0);
        col.load_queries(a.q, a.scale_log2, h);   // (clears the outputs)
        col.m = -__builtin_inff();
        col.l = 0.f;
      }
      x = y;
      i = 0;
      more = next(y);
      if (more) table.fetch(part, y, lane);
    }
  }
};

// ---- what the merge is told ----------------------------------------------------

// Where the pieces of a sequence's columns are: two ranges of units, the prefix's
// (units of KV head 0's segment from `off`, `head_off` further for each head, in
// workers of `run`; slots from `slot`, `head_slot` further for each head, `step` for
// each worker; its columns from `col` in a slot) and its own.
struct Describe {
  int4 units;   // off, head_off, units, run of the prefix (run 0: none)
  int4 slots;   // slot, head_slot, step, col
  int4 own;     // off, units, run (0: none), 0
};

__device__ __forceinline__ void describe(const SharedArgs& a, const SharedPlan& plan, int team_slot0, int few_slot0, int chunk,
                                         int lane) {
  const int s = 64 * chunk + lane, hkv = a.num_kv_heads;
  Describe d{int4{0, 0, 0, 0}, int4{0, 0, 1, 0}, int4{0, 0, 0, 0}};
  GroupSums gs;
#pragma unroll 1
  while (gs.chunk < a.prefix.rows) {
    const Groups x(a, gs, plan.team_run, lane);
    uint64_t some = __builtin_amdgcn_ballot_w64(x.kind != kNone && x.start < 64 * (chunk + 1) && x.start + x.count > 64 * chunk);
    while (some) {   // the prefixes whose groups reach into these sequences
      const int l = __builtin_ctzll(some);
      some &= some - 1;
      const int start = lane_value(x.start, l), units = lane_value(x.units, l), kind = lane_value(x.kind, l);
      const int base = lane_value(x.base, l), slot = lane_value(x.slot, l), wide = lane_value(x.wide, l);
      const int j = (s - start) << a.log2_group;
      if (s >= start && s < start + lane_value(x.count, l)) {
        d.units = int4{kind == kTeam ? 0 : base, units, units,
                       kind == kTeam ? lane_value(x.run, l) : (kind == kSingle ? plan.single_run : plan.few_run)};
        if (kind == kFew) d.slots = int4{few_slot0 + slot, 1, 1, j};
        else d.slots = int4{(kind == kTeam ? team_slot0 : 0) + slot + j / kPfCols, wide, kind == kTeam ? wide : kWaves, j & (kPfCols - 1)};
      }
    }
  }
  // the units of the sequences before this chunk
  int before = 0;
#pragma unroll 1
  for (int c = 0; c < 64 * chunk; c += 512) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int t = c + 64 * u + lane;
      before += units_of(t < 64 * chunk ? clamp_to(a.own.lens[t], 0, a.own.len_cap) : 0);
    }
  }
  SequenceSums ss{64 * chunk, hkv * last_lane(sum_scan(before))};
  const Sequences y(a, ss, lane);
  if (y.units > 0) d.own = int4{y.base, y.units, plan.own_run, 0};
  if (s < a.own.rows) reinterpret_cast<Describe*>(a.plan)[s] = d;
}

// ---- the kernel ---------------------------------------------------------------

template <typename T, bool ELASTIC, bool F8>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void shared_kernel(SharedArgs a) {
  __shared__ __attribute__((aligned(16))) char ring[kLdsBytes];
  Worker<T, ELASTIC, F8> worker(a, ring);
  const int lane = worker.lane, hkv = a.num_kv_heads;

  // the work of each kind
  GroupSums g;
#pragma unroll 1
  while (g.chunk < a.prefix.rows) Groups(a, g, 1, lane);
  int own_units = 0, own_rows = 0;   // (rows with tokens)
#pragma unroll 1
  for (int c = 0; c < a.own.rows; c += 512) {   // (8 loads in flight)
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int s = c + 64 * u + lane;
      const int n = units_of(s < a.own.rows ? clamp_to(a.own.lens[s], 0, a.own.len_cap) : 0);
      own_units += n;
      own_rows += n > 0 ? 1 : 0;
    }
  }
  own_units = hkv * last_lane(sum_scan(own_units));
  own_rows = last_lane(sum_scan(own_rows));
  const SharedPlan plan = divide_work(
      SharedWork{g.team_units, g.team_tiles, hkv * g.team_tiles, g.single_units, g.single_segments, g.few_units, g.few_segments, own_units, hkv * own_rows},
      (int)gridDim.x, a.min_units, F8);
  // slots: of the singles, of the teams, of the few
  const int team_slot0 = g.single_slots + kWaves * plan.single_workers;
  GroupSums t;
  if (plan.team_workers > 0) {
#pragma unroll 1
    while (t.chunk < a.prefix.rows) Groups(a, t, plan.team_run, lane);
  }
  const int few_slot0 = team_slot0 + t.team_slots;

  // What the merge needs, per sequence, written by the last workgroups, 64 sequences each.
  for (int c = gridDim.x - 1 - blockIdx.x; 64 * c < a.own.rows && worker.wave == 0; c += gridDim.x)
    describe(a, plan, team_slot0, few_slot0, c, lane);

  // a prefix, found by its kind and a unit (team: a worker); the search goes on where it ended
  struct {
    int p = -1, start, count, units, len, tiles, wide, base, slot, run, end;
  } at;
  GroupSums gs;
  auto find_prefix = [&](int pos, int kind) -> bool {
    if (at.p >= 0 && pos < at.end) return true;
#pragma unroll 1
    while (gs.chunk < a.prefix.rows) {
      const GroupSums before = gs;
      const Groups x(a, gs, plan.team_run, lane);
      const int all = hkv * x.units, end = x.base + (kind == kTeam ? (all + x.run - 1) / max(x.run, 1) * x.tiles : all);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(x.kind == kind && x.base <= pos && pos < end);
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
      at.run = lane_value(x.run, l);
      at.end = lane_value(end, l);
      gs = before;   // (the next prefix may lie in this chunk)
      return true;
    }
    return false;   // (lengths that changed under the launch)
  };

  const int w = blockIdx.x;
  if (w < plan.team_workers + plan.single_workers) {
    const bool team = w < plan.team_workers;
    // team workers in order of (prefix, team, tile), neighbours on one XCD (ids go round robin over the 8)
    const int q = plan.team_workers / 8, r = plan.team_workers % 8, xcd = w % 8;
    int id = team ? xcd * q + min(xcd, r) + w / 8 : w - plan.team_workers;
#pragma unroll 1
    for (bool again = true; again; ) {
      int tile = 0, slot0 = 0, pos, end;   // units: of the prefix (team), or of all singles
      if (team) {
        if (id >= t.team_workers || !find_prefix(id, kTeam)) break;
        const int m = (id - at.base) / at.tiles;
        tile = (id - at.base) - m * at.tiles;
        pos = m * at.run;
        end = min(hkv * at.units, pos + at.run);
        slot0 = team_slot0 + at.slot + m * at.wide;
        id += plan.team_workers;
      } else {
        pos = id * plan.single_run;
        end = min(g.single_units, pos + plan.single_run);
        again = false;
      }
#pragma unroll 1
      while (pos < end && (team || find_prefix(pos, kSingle))) {
        const int off = team ? pos : pos - at.base;
        const int first = tile * kTileCols;
        Piece pc;
        pc.row = at.p;
        pc.kvh = off / at.units;
        pc.len = at.len;
        pc.u0 = off - pc.kvh * at.units;
        pc.u1 = min(at.units, pc.u0 + (end - pos));
        pc.seq0 = at.start + (first >> a.log2_group);
        pc.columns = min((at.count << a.log2_group) - first, kTileCols);
        pc.slot = pc.kvh * at.wide + kWaves * tile + (team ? slot0 : at.slot + kWaves * id);
        worker.tile(pc);
        pos += pc.u1 - pc.u0;
      }
    }
    return;
  }

  // a wave's units: of the prefixes with few columns, or of the sequences
  const bool few = w < plan.team_workers + plan.single_workers + plan.few_workers;
  const int ww = (w - plan.team_workers - plan.single_workers - (few ? 0 : plan.few_workers)) * kWaves + worker.wave;
  int pos = ww * (few ? plan.few_run : plan.own_run);
  const int end = min(few ? g.few_units : own_units, pos + (few ? plan.few_run : plan.own_run));
  SequenceSums ss;
  auto find_sequence = [&](int u) -> bool {
    if (at.p >= 0 && u < at.end) return true;
#pragma unroll 1
    while (ss.chunk < a.own.rows) {
      const SequenceSums before = ss;
      const Sequences y(a, ss, lane);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(y.base <= u && u < y.base + hkv * y.units);
      if (!hit) continue;
      const int l = __builtin_ctzll(hit);
      at.p = before.chunk + l;
      at.len = lane_value(y.len, l);
      at.units = lane_value(y.units, l);
      at.base = lane_value(y.base, l);
      at.end = at.base + hkv * at.units;
      ss = before;
      return true;
    }
    return false;
  };
  const SharedPart part = few ? a.prefix : a.own;
  auto next = [&](Piece& x) -> bool {
    if (pos >= end || !(few ? find_prefix(pos, kFew) : find_sequence(pos))) return false;
    const int off = pos - at.base;
    x.row = at.p;
    x.len = at.len;
    x.kvh = off / at.units;
    x.u0 = off - x.kvh * at.units;
    x.u1 = min(at.units, x.u0 + min(64, end - pos));
    x.seq0 = few ? at.start : at.p;
    x.columns = (few ? at.count : 1) << a.log2_group;
    x.slot = (few ? few_slot0 + at.slot : at.p * hkv) + x.kvh + ww;
    pos += x.u1 - x.u0;
    return true;
  };
  worker.stream(part, next, few ? a.o_wide : a.o_own, few ? a.ml_wide : a.ml_own, few ? a.wide_slots : a.own_slots,
                few ? kPfCols : 1 << a.log2_group);
}

// ---- merge ---------------------------------------------------------------------
// A workgroup joins 32 columns (32 / G sequences of one KV head): lane l holds
// column l % 32, and wave w the chunks 4 w .. 4 w + 3 (2 each for l / 32).  Two
// memory round trips for up to 8 pieces of each part: the sequence's description,
// then maxima, sums and outputs together.
constexpr int kMergeWaves = 8, kAtOnce = 8;

// running (max, sum, outputs) of a column's chunks
struct Joined {
  float m = -__builtin_inff(), l = 0.f;
  f32x4 o[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
};

// Joins `n` pieces (per lane), `slot`, `slot + step`, ..., of slots with `width` columns, column `col`.
__device__ __forceinline__ void join(Joined& j, const float* os, const float* mls, int n, int slot, int step, int width, int col,
                                     int slots, int chunk) {
  const f32x4* op = reinterpret_cast<const f32x4*>(os);
  const float2* mp = reinterpret_cast<const float2*>(mls);
#pragma unroll 1
  for (int k0 = 0; __builtin_amdgcn_ballot_w64(k0 < n); k0 += kAtOnce) {
    float2 ml[kAtOnce];
    f32x4 x[kAtOnce][2];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int at = slot + (k0 + k) * step;
      ml[k] = make_float2(-__builtin_inff(), 0.f);
      x[k][0] = x[k][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (k0 + k < n && (unsigned)at < (unsigned)slots) {
        ml[k] = mp[(size_t)at * width + col];
#pragma unroll
        for (int i = 0; i < 2; ++i) x[k][i] = op[((size_t)at * 32 + chunk + 2 * i) * width + col];
      }
    }
    float top = j.m;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, ml[k].x);
    const float base = finite_or_zero(top);   // (no piece yet: every weight is 0)
    const float f = fast_exp2(j.m - base);
    j.l *= f;
#pragma unroll
    for (int i = 0; i < 2; ++i) j.o[i] *= f;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const float e = fast_exp2(ml[k].x - base);
      j.l += e * ml[k].y;
#pragma unroll
      for (int i = 0; i < 2; ++i) j.o[i] += e * x[k][i];
    }
    j.m = top;
  }
}

template <typename T>
__global__ __launch_bounds__(64 * kMergeWaves) void shared_merge_kernel(SharedArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.y;
  const int c = blockIdx.x * kPfCols + (lane & 31), chunk = 4 * wave + (lane >> 5);
  const int s = c >> a.log2_group, head = c & ((1 << a.log2_group) - 1);
  if (s >= a.own.rows) return;
  const Describe d = reinterpret_cast<const Describe*>(a.plan)[s];
  int wide_n = 0, wide_slot = 0, own_n = 0, own_slot = 0;
  if (d.units.w > 0) {
    const int off = d.units.x + kvh * d.units.y, w0 = off / d.units.w;
    wide_n = (off + d.units.z - 1) / d.units.w - w0 + 1;
    wide_slot = d.slots.x + kvh * d.slots.y + w0 * d.slots.z;
  }
  if (d.own.z > 0) {
    const int off = d.own.x + kvh * d.own.y, w0 = off / d.own.z;
    own_n = (off + d.own.y - 1) / d.own.z - w0 + 1;
    own_slot = s * a.num_kv_heads + kvh + w0;
  }
  Joined j;
  join(j, a.o_wide, a.ml_wide, wide_n, wide_slot, d.slots.z, kPfCols, d.slots.w + head, a.wide_slots, chunk);
  join(j, a.o_own, a.ml_own, own_n, own_slot, 1, 1 << a.log2_group, head, a.own_slots, chunk);
  const float inv = wide_n + own_n > 0 ? 1.0f / j.l : 0.f;   // (a sequence without any token: zeros)
  const size_t row = ((size_t)s * a.num_q_heads + (kvh << a.log2_group) + head) * kHeadDim;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const size_t idx = row + 4 * (chunk + 2 * i);
    store_pair<T>(a.out, idx, j.o[i][0] * inv, j.o[i][1] * inv, a.out_fp32);
    store_pair<T>(a.out, idx + 2, j.o[i][2] * inv, j.o[i][3] * inv, a.out_fp32);
  }
}

template <typename T, bool F8>
hipError_t launch_typed(const SharedArgs& a, bool elastic, hipStream_t st) {
  if (elastic) hipLaunchKernelGGL((shared_kernel<T, true, F8>), dim3(a.grid), dim3(64 * kWaves), 0, st, a);
  else hipLaunchKernelGGL((shared_kernel<T, false, F8>), dim3(a.grid), dim3(64 * kWaves), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int columns = a.own.rows << a.log2_group;
  hipLaunchKernelGGL((shared_merge_kernel<T>), dim3((columns + kPfCols - 1) / kPfCols, a.num_kv_heads),
                     dim3(64 * kMergeWaves), 0, st, a);
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
  *workgroups = 2 * cus;   // (74,880 B of LDS and at most 256 registers: two a CU)
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
