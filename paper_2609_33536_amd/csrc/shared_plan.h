// Parts of the shared-prefix decode that also compile for the host (internal
// header): the launch's arguments, and how its workgroups are divided.
#pragma once

#include <hip/hip_runtime.h>
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
  float scale_log2;
};

constexpr int kMaxSharedGrid = 512;

// Units and segments of each kind; a team's count once for each of its tiles.
struct SharedWork {
  int team_units, team_tiles, team_segments, single_units, single_segments, few_units, few_segments, own_units, own_segments;
};

// Workgroups of each kind, and the units that one takes (single), one of its 4
// waves (few, own), or a team of them takes of a prefix, at most (team).
struct SharedPlan {
  int team_workers, single_workers, few_workers, own_workers;
  int team_run, single_run, few_run, own_run;
};

// Divides `grid` workgroups (at least 4) over the kinds by their units and
// segments, weighted by what these cost a workgroup: a tile's unit is matrix work
// of 4 waves, the others' are bytes from HBM (half as many for 8-bit pools); a
// segment costs its start (table, queries, first loads) and its partials.
__host__ __device__ inline SharedPlan divide_work(const SharedWork& n, int grid, int min_units, bool bytes8) {
  const float stream = bytes8 ? 2.f : 3.f;
  const float cost[4] = {4.f * n.team_units + 16.f * n.team_segments, 4.f * n.single_units + 16.f * n.single_segments,
                         stream * n.few_units + 2.f * n.few_segments, stream * n.own_units + 2.f * n.own_segments};
  const float all = cost[0] + cost[1] + cost[2] + cost[3], share = all > 0.f ? grid / all : 0.f;
  int w[4], sum = 0, most = 0;
  for (int i = 0; i < 4; ++i) {
    w[i] = (int)(share * cost[i]);
    if (cost[i] > 0.f && w[i] == 0) w[i] = 1;
    sum += w[i];
    if (cost[i] > cost[most]) most = i;
  }
  if (all > 0.f) w[most] += grid - sum;   // (what rounding left over or took too much)
  auto run = [](int units, int workers, int least) -> int {
    const int r = workers > 0 ? (units + workers - 1) / workers : 1;
    return r > least ? r : least;
  };
  // teams: every prefix rounds its number of teams up, which adds at most its tiles to the workers
  const int spare = w[0] - n.team_tiles, teams = spare > w[0] / 2 ? spare : (w[0] + 1) / 2;
  return SharedPlan{w[0], w[1], w[2], w[3], run(n.team_units, teams, min_units), run(n.single_units, w[1], min_units),
                    run(n.few_units, 4 * w[2], min_units), run(n.own_units, 4 * w[3], 1)};
}

// Workgroups resident on the current device.
hipError_t shared_resident(int* workgroups);
// dtype: 0 bf16, 1 fp16, 3 8-bit.  Enqueues the attention and the merge.
hipError_t launch_shared(const SharedArgs& a, int dtype, bool elastic, hipStream_t st);

}  // namespace ekv
