// Parts of the shared-prefix decode that also compile for the host (internal
// header): the launch's arguments and sizes, how its workgroups are divided, and
// where the pieces' partials lie.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

namespace ekv {

// Rows of one block table: the prefixes, or the sequences' own tokens.
struct SharedPart {
  const uint16_t* pool;      // [NB][2][Hkv][16][128]
  const int32_t* lens;       // [rows]
  const int32_t* bt;         // [rows][max_blocks]
  const uint8_t* tags;       // [rows][max_blocks] or null
  const int32_t* bounds;     // [rows][2] or null
  int32_t rows, max_blocks, num_blocks, num_kv_heads;
  int32_t len_cap;           // lengths are clamped to this
};

struct SharedArgs {
  SharedPart prefix, own;
  const int32_t* starts;     // [prefix.rows + 1]: sequences starts[p] .. starts[p + 1] - 1 stand behind prefix p
  const uint16_t* q;         // [own.rows][Hq][128]
  void* out;                 // [own.rows][Hq][128]
  // scratch: where each sequence's pieces are, for the merge, then partials (max and sum; outputs) of pieces of 32 columns and of G columns
  int32_t* plan;
  float *ml_wide, *o_wide, *ml_own, *o_own;
  int32_t wide_slots, own_slots;
  int32_t num_kv_heads, num_q_heads, log2_group, out_fp32;
  int32_t grid;              // workgroups, at least 4 (one for each kind of work)
  int32_t min_units;         // fewest units of a prefix that a worker takes
  int32_t merge_ways;        // waves that divide a column's pieces in the merge: 1, 2, 4 or 8
  float scale_log2;
};

constexpr int kMaxSharedGrid = 512;
constexpr int kSharedWaves = 4;                  // of a workgroup
constexpr int kSharedCols = 32;                  // columns of a wave
constexpr int kSharedTile = kSharedWaves * kSharedCols;

// What a call is launched with, from the host's sizes alone.
struct SharedSize {
  int grid, min_units, merge_ways;
  int64_t wide_slots, own_slots;   // partials of 32 columns, and of G
};

// False if the flat spaces of units do not fit 32 bits.  Slots: at most one per 32
// columns (or part of 32) of a group and KV head, and 4 per workgroup for the segments
// that workers cut; likewise one per sequence and KV head.
inline bool size_shared(int64_t prefixes, int64_t rows, int64_t units_p, int64_t units_s, int64_t hkv, int64_t group,
                        SharedSize* l) {
  const int64_t columns = rows * group, groups = std::min<int64_t>(prefixes, rows);
  const int64_t tiles = columns / 128 + groups;
  const int64_t work_t = hkv * tiles * (units_p + 1), work_s = hkv * rows * (units_s + 1);   // (a segment's start counts too)
  if (work_t >= (1 << 30) || work_s >= (1 << 30) || columns * hkv >= (1 << 30) || prefixes >= (1 << 24)) return false;
  // The fewest units that a worker takes of a prefix, so that short prefixes leave the merge fewer
  // pieces: with 1 instead, 64 sequences behind 2048 tokens take 27.4 us (25.3), 8 behind 8192 23.7
  // (21.5), longer and shorter ones the same.
  l->min_units = (int)std::max<int64_t>(1, std::min<int64_t>(4, units_p / 16));
  const int64_t wanted = (work_t + hkv * groups * (units_p + 1) / 4 + work_s / 4) / l->min_units + 4;
  l->grid = (int)std::min<int64_t>(kMaxSharedGrid, wanted);
  // The merge: a workgroup takes 8 pieces a memory round trip.  Where a column may have more (at
  // most its units, or what is left of the workers for each segment), up to 8 waves divide them, as
  // long as the launch has at most one workgroup a compute unit.  With one wave always, 8 sequences
  // behind 32768 tokens take 68.5 us (39.1), 4 behind 512 14.2 (12.6); with up to two workgroups a
  // compute unit 16 prompts with samples take 66.8 (64.4).
  const int64_t pieces = std::min(units_p / l->min_units, 4 * l->grid / std::max<int64_t>(1, hkv * groups)) +
                         std::min(units_s, 4 * l->grid / std::max<int64_t>(1, hkv * rows));
  l->merge_ways = 1;
  while (l->merge_ways < 8 && pieces > 8 * l->merge_ways && (columns / 32 + 1) * hkv * 2 * l->merge_ways <= 256) l->merge_ways *= 2;
  l->wide_slots = hkv * (columns / 32 + groups) + columns / 32 + 4 * groups + 4 * l->grid;
  l->own_slots = hkv * rows + 4 * l->grid;
  return true;
}

// Units (few, own: and segments) of each kind; a team's count once for each of its tiles.
struct SharedWork {
  int team_units, team_tiles, team_segments, few_work, own_work;
};

// Workgroups of each kind, and the units that one of their waves takes (few, own), or
// a team of them at most (team): of one segment (aligned) or of a prefix's segments.
struct SharedPlan {
  int team_workers, few_workers, own_workers;
  int team_run, team_aligned, few_run, own_run;
};

// Divides `grid` workgroups (at least 4) over the kinds by their units and
// segments, weighted by what these cost a workgroup: a tile's unit is matrix work
// of 4 waves, the others' are bytes from HBM (half as many for 8-bit pools); a
// segment costs its start (table, queries, first loads) and its partials: one unit of
// a wave's stream, and of a tile 5, or 10 where first loads queue behind streams that
// use all of HBM's rate (16-bit pools: 64 sequences of up to 2048 behind 64 tokens
// 95.9 us at 5, 84.5 at 10; 8-bit, 44 of up to 2048 behind 256 tokens 41.0 and 48.4).
__host__ __device__ inline SharedPlan divide_work(const SharedWork& n, int grid, int min_units, bool bytes8) {
  const float stream = bytes8 ? 1.75f : 2.5f;
  const float team = 4.f * n.team_units + (bytes8 ? 20.f : 40.f) * n.team_segments;
  const float few = stream * n.few_work, own = stream * n.own_work;
  const float share = grid / fmaxf(1.f, team + few + own);
  int t = (int)(share * team), f = (int)(share * few), o = (int)(share * own);
  if (n.team_units > 0 && t == 0) t = 1;
  if (n.few_work > 0 && f == 0) f = 1;
  if (n.own_work > 0 && o == 0) o = 1;
  // Two tiles on one compute unit run slower than a tile beside streams: a few tiles more
  // than compute units are not worth it (three 8-bit prefixes of 16384 tokens and 44
  // sequences of up to 2048: 91.9 us, with the 273 tile workers of the weights alone 97.8).
  // Of 257 to 282 such tiles holding back was 2 to 12 % faster (6 of 6 batches), at 310 to 318
  // between 9 % faster (launches of 25 to 31 us) and 6 % slower (139 us); of more,
  // launches under 32 us would still gain 4 to 14 %, those of 100 us and more lose 4 to 23 %.
  constexpr int cus = kMaxSharedGrid / 2;
  const bool whole = t > cus && 4 * t < 5 * cus && f + o > 0;
  if (whole) t = cus;
  // (what rounding left over or took too much)
  const int rest = grid - t - f - o;
  if (t >= f && t >= o && !whole) t += rest;
  else if (f >= o) f += rest;
  else o += rest;
  SharedPlan p{t, f, o, 1, 0, 1, 1};
  if (n.few_work > 0) p.few_run = (n.few_work + 4 * f - 1) / (4 * f);
  if (p.few_run < min_units) p.few_run = min_units;
  if (n.own_work > 0) p.own_run = (n.own_work + 4 * o - 1) / (4 * o);
  if (n.team_units > 0) {
    // every prefix (or segment) rounds its number of teams up, which adds at most its tiles
    const int half = (t + 1) / 2, free = t - n.team_tiles > half ? t - n.team_tiles : half;
    p.team_run = (n.team_units + free - 1) / free;
    // One segment a team, unless that makes the run more than 5 units longer.  Over batches of 1
    // and 3 prefixes, runs up to 4 units longer were 0.4 to 12 % faster than shorter ones across
    // segments (12 of 12); 6 to 10 longer 1.5 % slower with 8-bit pools (7 of 10), and alike with
    // 16-bit ones (10 instead of 5 there: 0.98 to 1.035 of the time where it changes anything).
    if (t > n.team_segments) {
      const int run = (n.team_units + t - n.team_segments - 1) / (t - n.team_segments);
      if (run <= p.team_run + 5) {
        p.team_run = run;
        p.team_aligned = 1;
      }
    }
  }
  if (p.team_run < min_units) p.team_run = min_units;
  return p;
}

// ---- where the pieces are -------------------------------------------------------

enum Kind { kNone, kFew, kTeam };

// A prefix's columns: tiles of 128 and groups of 32 in them; up to 32 columns, or up to 32
// left over by the tiles, to a wave's stream (the last sequences' columns: a tile's unit
// costs the same for one column as for 128, and more than a stream's).
struct ColumnSplit {
  int tiles, wide, rest;
  __host__ __device__ inline ColumnSplit() {}
  __host__ __device__ inline explicit ColumnSplit(int columns) {
    rest = columns % kSharedTile <= kSharedCols ? columns % kSharedTile : 0;
    tiles = (columns - rest + kSharedTile - 1) / kSharedTile;
    wide = (columns - rest + kSharedCols - 1) / kSharedCols;
  }
};

// A prefix's teams: `spans` of `span` units, each cut into `cuts` runs of `run`.
struct Teams {
  int span, cuts, run;
  __host__ __device__ inline Teams(const SharedPlan& plan, int units, int hkv) {
    span = plan.team_aligned ? units : hkv * units;
    cuts = (span + plan.team_run - 1) / plan.team_run;
    run = cuts > 0 ? (span + cuts - 1) / cuts : 1;
  }
};

// Units with starts (few) or workers (team) of a prefix, and its slots (few: besides one for each worker).
struct Amounts {
  int work, slots;
  __host__ __device__ inline Amounts(const ColumnSplit& x, int units, const SharedPlan& plan, int kind, int hkv)
      : work(hkv * (units + 1)), slots(hkv) {
    if (kind == kTeam) {
      const Teams t(plan, units, hkv);
      work = (plan.team_aligned ? hkv : 1) * t.cuts * x.tiles;
      slots = (plan.team_aligned ? hkv * t.cuts : hkv + t.cuts) * x.wide;
    }
  }
};

// The first slot of team slots (the few's come first).
__host__ __device__ inline int first_team_slot(const SharedPlan& plan, int few_segments) {
  return few_segments + kSharedWaves * plan.few_workers;
}
// A tile's piece (its first wave's; the others' follow): `slot` the prefix's first, of team `team` on KV head kvh.
__host__ __device__ inline int tile_slot(const SharedPlan& plan, int slot, int wide, int team, int kvh, int tile) {
  return slot + (team + (plan.team_aligned ? 0 : kvh)) * wide + kSharedWaves * tile;
}
// A stream's piece: `slot` the prefix's or sequence's first, `worker` the wave's number in its kind.
__host__ __device__ inline int stream_slot(int slot, int kvh, int worker) { return slot + kvh + worker; }
// A sequence's own first slot.
__host__ __device__ inline int own_slot0(int sequence, int hkv) { return sequence * hkv; }

// Where the pieces of a sequence's columns are, for the merge: two ranges of units, the
// prefix's (units of KV head 0's segment from `off`, `head_off` further for each head, in
// workers of `run`; slots from `slot`, `head_slot` further for each head, `step` for
// each worker; its columns from `col` in a slot) and its own.
struct Describe {
  int4 units;   // off, head_off, units, run of the prefix (run 0: none)
  int4 slots;   // slot, head_slot, step, col
  int4 own;     // off, units, run (0: none), 0; a head's segment is units + 1 further than the one before
};

// The prefix's part, for a sequence whose first column is number `j` of the stream's (few) or
// the tiles' (team); base, slot: where the prefix's units (few) and slots begin.
__host__ __device__ inline void describe_columns(Describe& d, const SharedPlan& plan, int kind, int hkv, int units, int wide,
                                                 int base, int slot, int j) {
  if (kind == kFew) {
    d.units = int4{base + 1, units + 1, units, plan.few_run};
    d.slots = int4{slot, 1, 1, j};
  } else {
    const Teams t(plan, units, hkv);
    d.units = int4{0, plan.team_aligned ? t.cuts * t.run : units, units, t.run};
    d.slots = int4{slot + j / kSharedCols, plan.team_aligned ? 0 : wide, wide, j & (kSharedCols - 1)};
  }
}

// Pieces of one KV head: `n` of them, at slot, slot + step, ...
struct PieceSlots {
  int n, slot, step;
};
__host__ __device__ inline PieceSlots prefix_pieces(const Describe& d, int kvh) {
  if (d.units.w <= 0) return PieceSlots{0, 0, 1};
  const int off = d.units.x + kvh * d.units.y, w0 = off / d.units.w;
  return PieceSlots{(off + d.units.z - 1) / d.units.w - w0 + 1, d.slots.x + kvh * d.slots.y + w0 * d.slots.z, d.slots.z};
}
__host__ __device__ inline PieceSlots own_pieces(const Describe& d, int sequence, int hkv, int kvh) {
  if (d.own.z <= 0) return PieceSlots{0, 0, 1};
  const int off = d.own.x + kvh * (d.own.y + 1), w0 = off / d.own.z;
  return PieceSlots{(off + d.own.y - 1) / d.own.z - w0 + 1, stream_slot(own_slot0(sequence, hkv), kvh, w0), 1};
}

// Workgroups resident on the current device.
hipError_t shared_resident(int* workgroups);
// dtype: 0 bf16, 1 fp16, 3 8-bit.  Enqueues the attention and the merge.
hipError_t launch_shared(const SharedArgs& a, int dtype, bool elastic, hipStream_t st);

}  // namespace ekv
