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
  // scratch: the plan for the merge, then partials (max and sum; outputs) of pieces of 32 columns and of G columns
  int32_t* plan;
  float *ml_wide, *o_wide, *ml_own, *o_own;
  int32_t wide_slots, own_slots;
  int32_t num_kv_heads, num_q_heads, log2_group, out_fp32;
  int32_t grid;              // workgroups, at least 3 (one for each kind of work)
  int32_t min_units;         // fewest units a worker takes
  float scale_log2;
};

constexpr int kMaxSharedGrid = 512;

// Workgroups of each kind, and the units that a workgroup (tile) or one of its 4
// waves (few, own) takes.
struct SharedPlan {
  int tile_workers, few_workers, own_workers;
  int tile_run, few_run, own_run;
};

// Divides `grid` workgroups (at least 3) over the kinds by their units, weighted
// by what a unit costs: one of a tile holds 4 waves of matrix work, the others
// are bytes from HBM (half as many for 8-bit pools).
__host__ __device__ inline SharedPlan divide_work(int tile_units, int few_units, int own_units, int grid, int min_units,
                                                  bool bytes8) {
  const int64_t stream = bytes8 ? 2 : 3;
  const int64_t t = 4 * (int64_t)tile_units, f = stream * few_units, o = stream * own_units, all = t + f + o;
  SharedPlan p{0, 0, 0, 1, 1, 1};
  if (all == 0) return p;
  p.tile_workers = t ? (int)(grid * t / all) : 0;
  p.few_workers = f ? (int)(grid * f / all) : 0;
  if (t && p.tile_workers == 0) p.tile_workers = 1;
  if (f && p.few_workers == 0) p.few_workers = 1;
  p.own_workers = grid - p.tile_workers - p.few_workers;
  if (!o) {   // what is left over goes to the larger of the others
    (t >= f ? p.tile_workers : p.few_workers) += p.own_workers;
    p.own_workers = 0;
  } else if (p.own_workers < 1) {
    const int take = 1 - p.own_workers;
    (p.tile_workers >= p.few_workers ? p.tile_workers : p.few_workers) -= take;
    p.own_workers = 1;
  }
  auto run = [min_units](int units, int workers) -> int {
    const int r = workers > 0 ? (units + workers - 1) / workers : 1;
    return r > min_units ? r : min_units;
  };
  p.tile_run = run(tile_units, p.tile_workers);
  p.few_run = run(few_units, 4 * p.few_workers);
  p.own_run = run(own_units, 4 * p.own_workers);
  return p;
}

// Workgroups resident on the current device.
hipError_t shared_resident(int* workgroups);
// dtype: 0 bf16, 1 fp16, 3 8-bit.  Enqueues the attention and the merge.
hipError_t launch_shared(const SharedArgs& a, int dtype, bool elastic, hipStream_t st);

}  // namespace ekv
