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
// One launch works on three kinds of segments (a segment: one KV head of a prefix, or of
// a sequence's own tokens), each kind on workgroups of its own:
//   team   a prefix's query columns (sequence of the group, head of the KV head's G) in
//          tiles of 128: a team of workgroups, one for each tile, takes a run of a
//          segment's units, so that all of the team read the same K and V at the same
//          time, on one XCD.  In a tile 4 waves x 32 columns share every unit, pipelined
//          as in prefill.hip;
//   few    a prefix's columns if they are at most 32, or at most 32 left over by the
//          tiles: a wave streams the units alone;
//   own    a sequence's own tokens, G columns: likewise.
// The workgroups are divided between the kinds by the work that each has.  The units of
// few and own are one flat space each, in which a segment's start counts as a unit; a
// wave takes an equal run of it and crosses segments; a team stays in one segment where
// that makes its run little longer (divide_work), else it crosses the KV heads of its
// prefix.  Piece k of a segment is therefore made by worker w_first + k, and its slot of
// partials follows from segment and worker.
//
// What bounds it: behind a prefix of many columns matrix work (256 sequences of 64 query
// heads behind 32768 tokens: 0.94 PFLOP/s with P's remainder, a plain product reaches 1.22),
// otherwise HBM (64 sequences of 32 heads behind 8192 tokens, repeated: 187 MB in 39 us, 9
// of them before the stream is up, and 6 for the merge; 8 more on inputs in no cache);
// 8-bit pools the chain of a unit (widening, softmax, products).  64 sequences of 8192
// tokens each in rows of their own take 316 us.
#include <algorithm>
#include <atomic>

#include "prefill_device.h"
#include "shared_plan.h"
#include "wave_scan.h"

namespace ekv {
namespace {

constexpr int kWaves = kSharedWaves;
constexpr int kTileCols = kSharedTile;
static_assert(kSharedCols == kPfCols, "a wave's columns");
// LDS: 4 slots of K planes and 5 of V planes of a unit (tiles), or a unit's slot per wave (few, own).
constexpr int kVSlots = 5;
constexpr int kVRing = 4 * kPlanePf;
constexpr int kLdsRing = kVRing + kVSlots * kPlanePf;
constexpr int kLdsBytes = kLdsRing + kWaves * 64 * 16;   // and 16 bytes a lane (the first rows read)
static_assert(kLdsRing >= kWaves * kSlotPf, "a slot for every wave");
static_assert(2 * kLdsBytes <= 160 * 1024, "two workgroups a CU");

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return min(max(x, lo), hi); }
// The reference of a column all of whose scores so far are -inf: its weights are then 0, not NaN.
__device__ __forceinline__ float finite_or_zero(float m) { return m == -__builtin_inff() ? 0.f : m; }
__device__ __forceinline__ int units_of(int len) { return (len + 2 * kPage - 1) / (2 * kPage); }

// The lane, opaque: what follows from it is computed where it is used, not kept in
// registers from before a loop.
__device__ __forceinline__ int fresh(int lane) {
  asm volatile("" : "+v"(lane));
  return lane;
}
__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// Sum over the lanes, and each lane's sum of the lanes before it.  Most launches have
// one prefix (one lane that is not 0), which needs no scan.
struct LaneSum {
  int total, before;
  __device__ __forceinline__ explicit LaneSum(int x) : total(0), before(0) {
    const uint64_t some = __builtin_amdgcn_ballot_w64(x != 0);
    if (some & (some - 1)) {
      const int incl = sum_scan(x);
      before = incl - x;
      total = last_lane(incl);
    } else if (some) {
      total = lane_value(x, __builtin_ctzll(some));
    }
  }
};

// 64 prefixes, one a lane, as read: boundaries and length.
struct GroupRow {
  int start, end, len;
  __device__ __forceinline__ GroupRow(int s, int e, int l) : start(s), end(e), len(l) {}
  __device__ __forceinline__ GroupRow(const SharedArgs& a, int chunk, int lane) {
    const int p = chunk + lane;
    const bool in = p < a.prefix.rows;
    start = in ? clamp_to(a.starts[p], 0, a.own.rows) : a.own.rows;
    end = in ? clamp_to(a.starts[p + 1], 0, a.own.rows) : a.own.rows;
    len = in ? clamp_to(a.prefix.lens[p], 0, a.prefix.len_cap) : 0;
  }
};

// What follows from a prefix's sequences and length.
struct Shape : ColumnSplit {
  int start, count, units, len;            // (units: 0 without any sequence)
  __device__ __forceinline__ Shape() {}
  __device__ __forceinline__ Shape(int start_, int end, int len_, int log2_group) : start(start_), len(len_) {
    count = len > 0 ? end - start : 0;
    units = count > 0 ? units_of(len) : 0;
    static_cast<ColumnSplit&>(*this) = ColumnSplit(count << log2_group);
  }
  __device__ __forceinline__ bool has(int kind) const { return kind == kTeam ? tiles > 0 : rest > 0; }
  // the first sequence of the stream's columns
  __device__ __forceinline__ int rest_start(int log2_group) const { return start + count - (rest >> log2_group); }
};

// Of 64 prefixes.  The group boundaries are clamped into the batch and made
// nondecreasing (`from`: the boundary so far, advanced), so that groups never overlap.
struct Groups : Shape {
  __device__ __forceinline__ Groups(const SharedArgs& a, const GroupRow& r, int& from) {
    int s = r.start, e = r.end;
    if (__builtin_amdgcn_ballot_w64(e < s || s < from)) {   // (boundaries that fall)
      s = max(max_scan(s), from);
      e = max(s, e);
      from = last_lane(max_scan(e));
    } else {
      from = last_lane(e);
    }
    static_cast<Shape&>(*this) = Shape(s, e, r.len, a.log2_group);
  }
};

// Where the work and the slots of 64 prefixes of one kind begin.  `work` and `slots`
// count those before, and are advanced.
struct Places {
  int base, end, slot;
  __device__ __forceinline__ Places(const Groups& x, const SharedPlan& plan, int kind, int hkv, int& work, int& slots) {
    const Amounts n(x, x.units, plan, kind, hkv);
    const bool mine = x.has(kind);
    const LaneSum sw(mine ? n.work : 0), sn(mine ? n.slots : 0);
    base = work + sw.before;
    end = mine ? base + n.work : base;
    slot = slots + sn.before;
    work += sw.total;
    slots += sn.total;
  }
};

// One prefix and its place.
struct Group : Shape {
  int p, base, end, slot;
  __device__ __forceinline__ Group() {}
  __device__ __forceinline__ Group(const Groups& x, const Places& at, int c0, int l) {
    p = c0 + l;
    start = lane_value(x.start, l);
    count = lane_value(x.count, l);
    units = lane_value(x.units, l);
    len = lane_value(x.len, l);
    rest = lane_value(x.rest, l);
    tiles = lane_value(x.tiles, l);
    wide = lane_value(x.wide, l);
    base = lane_value(at.base, l);
    end = lane_value(at.end, l);
    slot = lane_value(at.slot, l);
  }
};

// A row's units in the flat space of its kind, for one KV head.
__device__ __forceinline__ int work_of(int len) { return len > 0 ? units_of(len) + 1 : 0; }

// 64 sequences, one a lane: their own tokens and where their units begin.
struct SequenceSums {
  int chunk = 0, units = 0;
};
__device__ __forceinline__ int own_length(const SharedArgs& a, int s) {
  return s < a.own.rows ? clamp_to(a.own.lens[s], 0, a.own.len_cap) : 0;
}
struct Sequences {
  int len, units, base;
  // (length: of sequence chunk + lane)
  __device__ __forceinline__ Sequences(const SharedArgs& a, SequenceSums& sums, int length) : len(length) {
    units = units_of(len);
    const int n = a.num_kv_heads * work_of(len), incl = sum_scan(n);
    base = sums.units + incl - n;
    sums.chunk += 64;
    sums.units += last_lane(incl);
  }
};

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

  __device__ __forceinline__ Worker(const SharedArgs& a_, char* ring_, int wave_, int lane_)
      : a(a_), ring(ring_), wave(wave_), lane(lane_), h(lane_ >> 5) {}

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
    const Stager<F8> stager(lane, a.num_kv_heads);
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
    // what landed of K of unit u and V of unit u - 1 (this wave's quarters), and its words in place
    u32x4 raw_k, raw_v;
    auto take = [&](int u) {
      raw_k = stager.landed_plane(ring + k_slot(u), is_base(u), wave, lane);
      raw_v = stager.landed_plane(ring + kVRing + v_stage, is_base(u - 1), wave, lane);
    };
    auto stage = [&](int u) {
      char* at = ring + kVRing + next_v(v_stage);
      stager.widen_plane(ring + k_slot(u), is_base(u), wave, raw_k);
      stager.widen_plane(at, is_base(u - 1), wave, raw_v);
      stager.clear_tail(at, wave, 2 * kPage * (x.u0 + u - 1), x.len);
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
    raw_k = stager.landed_plane(ring + k_slot(0), is_base(0), wave, lane);
    stager.widen_plane(ring + k_slot(0), is_base(0), wave, raw_k);
    take(1);
    stage(1);
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
        landed();
        take(i + 2);
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
      } else {
        landed();
        take(i + 2);
      }
      stage(i + 2);
    }
    wait_loads<0>();   // no load may land in a slot of the next piece, or after the workgroup has ended
    products();
    if (active) store(col, a.o_wide, a.ml_wide, x.slot + wave, a.wide_slots, kPfCols);
    barrier();         // every wave is done with the rings
  }

  // One wave's columns over a run of units, alone, in the wave's own slot of LDS.
  // `next` gives the run's pieces one after the other, at most 64 units each, and
  // is asked two ahead: while piece x is worked on, the block table of y is in
  // registers, or y's first unit in flight and the table of z on its way.  A piece's
  // first unit is loaded and its queries read as soon as the last unit before it
  // has left the slot and the query registers, so that the wave's stream of loads does
  // not stop between segments.
  template <typename Next>
  __device__ __forceinline__ void stream(const SharedPart& part, Next next, float* o, float* ml, int slots, int width) {
    ColumnState<T> col;
    const Stager<F8> stager(lane, a.num_kv_heads);
    char* slot = ring + wave * kSlotPf;
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(lds_ptr)slot);
    const uint32_t k_at = k_read_offset(lane), v_at = v_read_offset(lane);
    UnitTable<ELASTIC, F8> table(part);
    Piece x, y;
    if (!next(x)) return;
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
    bool more = next(y);      // y: the piece after x
    if (more) table.fetch(part, y, lane);
    int i = 0;                // unit of the piece
#pragma unroll 1
    while (true) {
      const int key0 = 2 * kPage * (x.u0 + i);
      wait_loads<0>();
      if (F8 || base) {   // (all is read before any of it is widened: one LDS round trip)
        u32x4 raw[4][2];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int pl = 0; pl < 2; ++pl) raw[q][pl] = stager.landed_plane(slot + pl * kPlanePf, base, q, lane);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int pl = 0; pl < 2; ++pl) stager.widen_plane(slot + pl * kPlanePf, base, q, raw[q][pl]);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) stager.clear_tail(slot + kPlanePf, q, key0, x.len);
      u32x4 k[8], v[2][4], hi[2], lo[2];
      read_k(slot + k_at, k);
      read_v(slot + v_at, v);
      f32x16 sc = col.scores(k);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot has been read
      const bool last = x.u0 + ++i == x.u1;   // the piece's last unit
      const float c = col.mask(sc, key0, h);
      Piece z;
      bool beyond = false;
      if (!last) {
        issue(i);
      } else if (more) {
        table.enter(lane, y);
        issue(0);
        beyond = next(z);
        if (beyond) table.fetch(part, z, lane);
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
      y = z;
      more = beyond;
      i = 0;
    }
  }
};

// ---- what the merge is told ----------------------------------------------------

// The prefix's part, for the sequences of chunk `chunk` (one a lane) that stand behind
// prefix g in its columns of one kind; slot0: that kind's first slot.
__device__ __forceinline__ void describe_prefix(Describe& d, const SharedArgs& a, const SharedPlan& plan, const Group& g, int kind,
                                                int slot0, int chunk, int lane) {
  const int s = 64 * chunk + lane, rest = g.rest_start(a.log2_group);
  const int first = kind == kFew ? rest : g.start;
  if (s < first || s >= (kind == kFew ? g.start + g.count : rest)) return;
  describe_columns(d, plan, kind, a.num_kv_heads, g.units, g.wide, g.base, slot0 + g.slot, (s - first) << a.log2_group);
}
// Those of one kind among the 64 prefixes x whose groups reach into these sequences.
__device__ __forceinline__ void describe_prefixes(Describe& d, const SharedArgs& a, const SharedPlan& plan, const Groups& x,
                                                  const Places& at, int kind, int slot0, int chunk, int lane) {
  uint64_t some = __builtin_amdgcn_ballot_w64(x.has(kind) && x.start < 64 * (chunk + 1) && x.start + x.count > 64 * chunk);
#pragma unroll 1
  while (some) {
    const int l = __builtin_ctzll(some);
    some &= some - 1;
    describe_prefix(d, a, plan, Group(x, at, 0, l), kind, slot0, chunk, lane);
  }
}
// The sequences' own part.
__device__ __forceinline__ void describe_own(Describe& d, const SharedArgs& a, const SharedPlan& plan, int chunk, int lane) {
  int before = 0;   // the units of the sequences before this chunk
#pragma unroll 1
  for (int c = 0; c < 64 * chunk; c += 512) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int t = c + 64 * u + lane;
      before += work_of(t < 64 * chunk ? own_length(a, t) : 0);
    }
  }
  SequenceSums ss{64 * chunk, a.num_kv_heads * last_lane(sum_scan(before))};
  const Sequences y(a, ss, own_length(a, 64 * chunk + lane));
  if (y.units > 0) d.own = int4{y.base + 1, y.units, plan.own_run, 0};
}

// ---- the kernel ---------------------------------------------------------------

// The launch's arguments, through an opaque pointer to them: a field is loaded where it
// is used (a scalar load that hits the cache), not kept in scalar registers, of which
// there are too few, from the kernel's start.
__device__ __forceinline__ const SharedArgs& arguments() {
  auto p = (const __attribute__((address_space(4))) SharedArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const SharedArgs*)p;
}

template <typename T, bool ELASTIC, bool F8>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void shared_kernel(SharedArgs) {
  const SharedArgs& a = arguments();
  __shared__ __attribute__((aligned(16))) char ring[kLdsBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hkv = a.num_kv_heads;

  // (the first 64 prefixes and sequences are read once and kept in LDS, a copy for every wave)
  int4* rows0 = reinterpret_cast<int4*>(ring + kLdsRing) + 64 * wave + lane;
  int own_work;   // units and starts of all sequences
  {
    const GroupRow r(a, 0, lane);
    const int len0 = own_length(a, lane);
    *rows0 = int4{r.start, r.end, r.len, len0};
    own_work = work_of(len0);
  }
#pragma unroll 1
  for (int c = 64; c < a.own.rows; c += 512) {   // (8 loads in flight)
#pragma unroll
    for (int u = 0; u < 8; ++u) own_work += work_of(own_length(a, c + 64 * u + lane));
  }
  own_work = hkv * last_lane(sum_scan(own_work));

  // One loop scans the prefixes and works, so that the code of either is there once (a
  // launch starts with a cold instruction cache): pass 0 adds up the work of each kind
  // and divides the workers; pass 1 describes sequences to the merge and finds this
  // worker's first prefix; later ones find the next prefix.
  SharedPlan plan{};
  int kind = kNone;              // of this worker (kNone: a wave for the sequences' own tokens)
  int id = 0, pos = 0, end = 0;  // its number in its kind (few, own: this wave's); its units (team: its number)
  int few_work = 0, team_units = 0, team_tiles = 0, few_segments = 0, team_slot0 = 0;   // (the few's slots come first)
#pragma unroll 1
  for (int pass = 0;; ++pass) {
    const SharedArgs& a = arguments();
    Group at;
    bool found = pass > 0 && kind == kNone;
    const int chunk = gridDim.x - 1 - blockIdx.x;   // the last workgroups describe 64 sequences each
    const bool describes = pass == 1 && wave == 0 && 64 * chunk < a.own.rows;
    Describe d{int4{0, 0, 0, 0}, int4{0, 0, 1, 0}, int4{0, 0, 0, 0}};
    int from = 0, work = 0, slots = 0, other_work = 0, other_slots = 0;
    const bool one = a.prefix.rows == 1;   // (in scalars, without a scan)
    if (one) {
      const int4 v = *rows0;
      const int start = lane_value(v.x, 0);
      static_cast<Shape&>(at) = Shape(start, max(start, lane_value(v.y, 0)), lane_value(v.z, 0), a.log2_group);
      at.p = at.base = at.slot = 0;
      if (pass == 0) {
        few_work = at.has(kFew) ? hkv * (at.units + 1) : 0;
        few_segments = at.has(kFew) ? hkv : 0;
        team_tiles = at.tiles;
        team_units = hkv * at.tiles * at.units;
      } else {
        if (kind != kNone && at.has(kind)) {
          at.end = Amounts(at, at.units, plan, kind, hkv).work;
          found = pos < at.end;
        }
        if (describes) {
          if (at.has(kTeam)) describe_prefix(d, a, plan, at, kTeam, team_slot0, chunk, lane);
          if (at.has(kFew)) describe_prefix(d, a, plan, at, kFew, 0, chunk, lane);
        }
      }
    }
#pragma unroll 1
    for (int c0 = one ? 1 : 0; c0 < a.prefix.rows && (pass < 2 || !found); c0 += 64) {
      GroupRow r(0, 0, 0);
      if (c0 == 0) {
        const int4 v = *rows0;
        r = GroupRow(v.x, v.y, v.z);
      } else {
        r = GroupRow(a, c0, lane);
      }
      const Groups x(a, r, from);
      if (pass == 0) {
        few_work += LaneSum(x.has(kFew) ? hkv * (x.units + 1) : 0).total;
        few_segments += hkv * __builtin_popcountll(__builtin_amdgcn_ballot_w64(x.has(kFew)));
        team_units += LaneSum(hkv * x.tiles * x.units).total;
        team_tiles += LaneSum(x.tiles).total;
        continue;
      }
      if (describes) {
        const int other = kind == kTeam ? kFew : kTeam;   // (own workers: both kinds, one here and one below)
        const Places y(x, plan, other, hkv, other_work, other_slots);
        describe_prefixes(d, a, plan, x, y, other, other == kTeam ? team_slot0 : 0, chunk, lane);
      }
      const int mine = kind == kNone ? kFew : kind;
      const Places y(x, plan, mine, hkv, work, slots);
      if (describes) describe_prefixes(d, a, plan, x, y, mine, mine == kTeam ? team_slot0 : 0, chunk, lane);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(x.has(mine) && y.base <= pos && pos < y.end);
      if (found || !hit) continue;
      found = true;
      at = Group(x, y, c0, __builtin_ctzll(hit));
    }
    if (pass == 0) {
      plan = divide_work(SharedWork{team_units, team_tiles, hkv * team_tiles, few_work, own_work},
                         (int)gridDim.x, a.min_units, F8);
      team_slot0 = first_team_slot(plan, few_segments);
      id = blockIdx.x;
      if (id < plan.team_workers) {
        // team workers in order of (prefix, segment, run, tile), neighbours on one XCD (ids go round robin over the 8)
        const int q = plan.team_workers / 8, r = plan.team_workers % 8;
        kind = kTeam;
        id = id % 8 * q + min(id % 8, r) + id / 8;
        pos = id;
        end = pos + 1;
      } else {
        id -= plan.team_workers;
        kind = id < plan.few_workers ? kFew : kNone;
        if (kind == kNone) id -= plan.few_workers;
        id = id * kWaves + wave;
        const int run = kind == kFew ? plan.few_run : plan.own_run;
        pos = id * run;
        end = min(kind == kFew ? few_work : own_work, pos + run);
      }
      continue;
    }
    if (describes) {
      describe_own(d, a, plan, chunk, lane);
      if (64 * chunk + lane < a.own.rows) reinterpret_cast<Describe*>(a.plan)[64 * chunk + lane] = d;
    }
    if (!found || pos >= end) return;

    if (kind == kTeam) {
      const SharedArgs& a = arguments();
      const Teams t(plan, at.units, hkv);
      const int team = (pos - at.base) / at.tiles, tile = (pos - at.base) - team * at.tiles;
      const int k = team / t.cuts, first = tile * kTileCols;   // span; first column
      int u = k * t.span + (team - k * t.cuts) * t.run;
      const int u_end = min((k + 1) * t.span, u + t.run);
#pragma unroll 1
      while (u < u_end) {
        Piece pc;
        pc.row = at.p;
        pc.kvh = u / at.units;
        pc.len = at.len;
        pc.u0 = u - pc.kvh * at.units;
        pc.u1 = min(at.units, pc.u0 + (u_end - u));
        pc.seq0 = at.start + (first >> a.log2_group);
        pc.columns = min((at.count << a.log2_group) - at.rest - first, kTileCols);
        pc.slot = tile_slot(plan, team_slot0 + at.slot, at.wide, team, pc.kvh, tile);
        Worker<T, ELASTIC, F8>(arguments(), ring, wave, fresh(lane)).tile(pc);
        u += pc.u1 - pc.u0;
      }
      pos += plan.team_workers;   // (more of the prefixes' tiles than workers: another round)
      end = pos + 1;
      continue;
    }

    // a wave's units of one prefix, or of the sequences
    const bool few = kind == kFew;
    int u = pos;
    const int u_end = few ? min(end, at.end) : end;
    int seqs = 0, lane_at = 0, lens = rows0->w;   // own: the chunk of sequences at hand, the one in it, the lengths
    if (!few) {
      SequenceSums ss;
      uint64_t hit = 0;
#pragma unroll 1
      while (!hit && ss.chunk < a.own.rows) {
        seqs = ss.chunk;
        if (seqs > 0) lens = own_length(a, seqs + lane);
        const Sequences y(a, ss, lens);
        hit = __builtin_amdgcn_ballot_w64(y.base <= u && u < y.base + hkv * work_of(lens));
        if (!hit) continue;
        lane_at = __builtin_ctzll(hit);
        at.base = lane_value(y.base, lane_at);
        at.end = at.base;   // (set below)
      }
      if (!hit) return;     // (lengths that changed under the launch)
    }
    bool enter = !few;
    auto next = [&](Piece& x) -> bool {
      if (u >= u_end) return false;
      if (!few && (enter || u >= at.end)) {
        if (!enter) {       // the next sequence that has tokens
          at.base = at.end;
          uint64_t left = lane_at == 63 ? 0 : __builtin_amdgcn_ballot_w64(lens > 0) & (~0ull << (lane_at + 1));
#pragma unroll 1
          while (!left) {
            seqs += 64;
            if (seqs >= a.own.rows) return false;
            lens = own_length(a, seqs + lane);
            left = __builtin_amdgcn_ballot_w64(lens > 0);
          }
          lane_at = __builtin_ctzll(left);
        }
        enter = false;
        at.p = at.start = seqs + lane_at;
        at.len = lane_value(lens, lane_at);
        at.units = units_of(at.len);
        at.end = at.base + hkv * (at.units + 1);
        at.rest = 1 << a.log2_group;
        at.slot = own_slot0(at.p, hkv);
      }
      x.row = at.p;
      x.len = at.len;
      x.kvh = (u - at.base) / (at.units + 1);
      x.u0 = u - at.base - x.kvh * (at.units + 1) - 1;
      if (x.u0 < 0) {       // the segment's start
        x.u0 = 0;
        if (++u >= u_end) return false;
      }
      x.u1 = min(at.units, x.u0 + min(64, u_end - u));
      x.seq0 = few ? at.rest_start(a.log2_group) : at.start;
      x.columns = at.rest;
      x.slot = stream_slot(at.slot, x.kvh, id);
      u += x.u1 - x.u0;
      return true;
    };
    Worker<T, ELASTIC, F8>(arguments(), ring, wave, fresh(lane)).stream(few ? a.prefix : a.own, next, few ? a.o_wide : a.o_own, few ? a.ml_wide : a.ml_own,
                  few ? a.wide_slots : a.own_slots, few ? kPfCols : 1 << a.log2_group);
    if (!few) return;
    pos = u_end;
  }
}

// ---- merge ---------------------------------------------------------------------
// A workgroup joins 32 columns (32 / G sequences of one KV head): lane l holds
// column l % 32, and wave w the chunks 4 w .. 4 w + 3 (2 each for l / 32).  Two
// memory round trips for up to 8 pieces of the prefix and 4 of the sequence's own: the
// sequence's description, then maxima, sums and outputs together.
constexpr int kMergeWaves = 8;

// running (max, sum, outputs) of a column's chunks
struct Joined {
  float m = -__builtin_inff(), l = 0.f;
  f32x4 o[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
};

// N pieces of a column, loaded together: those from k0 on of `n` (per lane) at `slot`,
// `slot + step`, ..., of slots with `width` columns, column `col`.
template <int N>
struct Pieces {
  float2 ml[N];
  f32x4 x[N][2];
  __device__ __forceinline__ Pieces(const float* os, const float* mls, int k0, int n, int slot, int step, int width, int col,
                                    int slots, int chunk) {
    const f32x4* op = reinterpret_cast<const f32x4*>(os);
    const float2* mp = reinterpret_cast<const float2*>(mls);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int at = slot + (k0 + k) * step;
      ml[k] = make_float2(-__builtin_inff(), 0.f);
      x[k][0] = x[k][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (k0 + k < n && (unsigned)at < (unsigned)slots) {
        ml[k] = mp[(size_t)at * width + col];
#pragma unroll
        for (int i = 0; i < 2; ++i) x[k][i] = op[((size_t)at * 32 + chunk + 2 * i) * width + col];
      }
    }
  }
  __device__ __forceinline__ void join(Joined& j) const {
    float top = j.m;
#pragma unroll
    for (int k = 0; k < N; ++k) top = fmaxf(top, ml[k].x);
    const float base = finite_or_zero(top);   // (no piece yet: every weight is 0)
    const float f = fast_exp2(j.m - base);
    j.l *= f;
#pragma unroll
    for (int i = 0; i < 2; ++i) j.o[i] *= f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float e = fast_exp2(ml[k].x - base);
      j.l += e * ml[k].y;
#pragma unroll
      for (int i = 0; i < 2; ++i) j.o[i] += e * x[k][i];
    }
    j.m = top;
  }
};

// `ways` (1, 2, 4 or 8) waves divide a column's pieces between them and join theirs
// through LDS; a workgroup then has 8 / ways waves' chunks, and grid z is ways.
template <typename T>
__global__ __launch_bounds__(64 * kMergeWaves) void shared_merge_kernel(SharedArgs a) {
  __shared__ float parts[kMergeWaves][10][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.y, ways = gridDim.z, way = wave & (ways - 1);
  const int c = blockIdx.x * kPfCols + (lane & 31);
  const int chunk = 4 * ((wave + kMergeWaves * blockIdx.z) / ways) + (lane >> 5);
  const int s = c >> a.log2_group, head = c & ((1 << a.log2_group) - 1);
  const bool ok = s < a.own.rows;
  int wide_n = 0, wide_slot = 0, own_n = 0, own_slot = 0, step = 1, col = 0;
  if (ok) {
    const Describe d = reinterpret_cast<const Describe*>(a.plan)[s];
    const PieceSlots w = prefix_pieces(d, kvh), o = own_pieces(d, s, a.num_kv_heads, kvh);
    wide_n = w.n;
    wide_slot = w.slot;
    step = w.step;
    col = d.slots.w + head;
    own_n = o.n;
    own_slot = o.slot;
  }
  const int all_n = wide_n + own_n;
  // this way's pieces: every `ways`-th from `way` on
  wide_slot += way * step;
  own_slot += way;
  wide_n = (wide_n - way + ways - 1) / ways;
  own_n = (own_n - way + ways - 1) / ways;
  Joined j;
  constexpr int kWide = 8, kOwn = 4;
#pragma unroll 1
  for (int w0 = 0, o0 = 0; __builtin_amdgcn_ballot_w64(w0 < wide_n || o0 < own_n); w0 += kWide, o0 += kOwn) {
    const Pieces<kWide> w(a.o_wide, a.ml_wide, w0, wide_n, wide_slot, step * ways, kPfCols, col, a.wide_slots, chunk);
    const Pieces<kOwn> o(a.o_own, a.ml_own, o0, own_n, own_slot, ways, 1 << a.log2_group, head, a.own_slots, chunk);
    w.join(j);
    o.join(j);
  }
  if (ways > 1) {
    if (way > 0) {
      parts[wave][0][lane] = j.m;
      parts[wave][1][lane] = j.l;
#pragma unroll
      for (int i = 0; i < 8; ++i) parts[wave][2 + i][lane] = j.o[i >> 2][i & 3];
    }
    __syncthreads();
    if (way > 0) return;
#pragma unroll 1
    for (int w = wave + 1; w < wave + ways; ++w) {
      const float m = parts[w][0][lane], top = fmaxf(j.m, m), base = finite_or_zero(top);
      const float f = fast_exp2(j.m - base), e = fast_exp2(m - base);
      j.l = j.l * f + parts[w][1][lane] * e;
#pragma unroll
      for (int i = 0; i < 8; ++i) j.o[i >> 2][i & 3] = j.o[i >> 2][i & 3] * f + parts[w][2 + i][lane] * e;
      j.m = top;
    }
  }
  if (!ok) return;
  const float inv = all_n > 0 ? 1.0f / j.l : 0.f;   // (a sequence without any token: zeros)
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
  hipLaunchKernelGGL((shared_merge_kernel<T>), dim3((columns + kPfCols - 1) / kPfCols, a.num_kv_heads, a.merge_ways),
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
  *workgroups = 2 * cus;   // (78,976 B of LDS and at most 256 registers: two a CU)
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
