// Parts of the shared-prefix decode that also compile for the host (internal
// header): the launch's arguments, and how its workgroups are divided.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

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
// 95.9 us at 5, 84.5 at 10; 8-bit, 55 of up to 2048 behind 256 tokens 41.0 and 48.4).
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
  // than compute units are not worth it (three 8-bit prefixes of 16384 tokens and 55
  // sequences of up to 2048: 91.9 us, with the 273 tile workers of the weights alone 97.8).
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
    if (t > n.team_segments) {
      const int run = (n.team_units + t - n.team_segments - 1) / (t - n.team_segments);
      if (run <= p.team_run + 5) {   // (a start costs a worker what 5 units do)
        p.team_run = run;
        p.team_aligned = 1;
      }
    }
  }
  if (p.team_run < min_units) p.team_run = min_units;
  return p;
}

// Workgroups resident on the current device.
hipError_t shared_resident(int* workgroups);
// dtype: 0 bf16, 1 fp16, 3 8-bit.  Enqueues the attention and the merge.
hipError_t launch_shared(const SharedArgs& a, int dtype, bool elastic, hipStream_t st);

}  // namespace ekv
