// Random batches through divide_work(): every workgroup has a kind, every kind's work is
// covered, and the slots that the pieces take fit the workspace's count of them.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "shared_plan.h"

using namespace ekv;

int main() {
  std::mt19937 rng(1);
  auto in = [&](int lo, int hi) { return (int)(lo + rng() % (unsigned)(hi - lo + 1)); };
  long checked = 0, bad = 0;
  for (int it = 0; it < 100000; ++it) {
    const int hkv = 1 << in(0, 4), group = 1 << in(0, 4), prefixes = in(0, 3) ? in(1, 4) : in(1, 40);
    std::vector<int> count(prefixes), len(prefixes);
    int rows = in(0, 3), longest = 1;
    for (int p = 0; p < prefixes; ++p) {
      count[p] = in(0, 4) ? in(0, 1 << in(0, 8)) : 0;
      len[p] = in(0, 8) ? in(1, 1 << in(1, 15)) : 0;
      rows += count[p];
      longest = std::max(longest, len[p]);
    }
    if (rows == 0) continue;
    longest += in(0, 100);
    const int own = in(1, 2000);
    // as the entry point sizes a call
    const long columns = (long)rows * group, groups = std::min(prefixes, rows);
    const long units_p = ((longest + 15) / 16 + 1) / 2, units_s = ((own + 15) / 16 + 1) / 2;
    const long work_t = hkv * (columns / 128 + groups) * (units_p + 1), work_s = (long)hkv * rows * (units_s + 1);
    if (work_t >= (1 << 30) || work_s >= (1 << 30)) continue;
    const int min_units = (int)std::max(1L, std::min(4L, units_p / 16));
    const long wanted = (work_t + hkv * groups * (units_p + 1) / 4 + work_s / 4) / min_units + 4;
    const int sized = (int)std::min<long>(kMaxSharedGrid, wanted), grid = std::max(4, std::min(sized, in(0, 1) ? kMaxSharedGrid : in(8, kMaxSharedGrid)));
    const long wide_slots = hkv * (columns / 32 + groups) + columns / 32 + 4 * groups + 4 * sized, own_slots = (long)hkv * rows + 4 * sized;
    // as the kernel counts the work
    SharedWork w{0, 0, 0, 0, 0};
    for (int r = 0; r < rows; ++r) {
      const int n = in(0, own);
      w.own_work += n > 0 ? hkv * ((n + 31) / 32 + 1) : 0;
    }
    std::vector<int> tiles(prefixes), wide(prefixes), units(prefixes);
    int few_segments = 0;
    for (int p = 0; p < prefixes; ++p) {
      const int c = len[p] > 0 ? count[p] * group : 0, rest = c % 128 <= 32 ? c % 128 : 0;
      units[p] = c > 0 ? (len[p] + 31) / 32 : 0;
      tiles[p] = (c - rest + 127) / 128;
      wide[p] = (c - rest + 31) / 32;
      if (rest > 0) {
        w.few_work += hkv * (units[p] + 1);
        few_segments += hkv;
      }
      w.team_tiles += tiles[p];
      w.team_units += hkv * tiles[p] * units[p];
    }
    w.team_segments = hkv * w.team_tiles;
    for (int bytes8 = 0; bytes8 < 2; ++bytes8) {
      const SharedPlan p = divide_work(w, grid, min_units, bytes8 != 0);
      bool ok = p.team_workers >= 0 && p.few_workers >= 0 && p.own_workers >= 0 &&
                p.team_workers + p.few_workers + p.own_workers == grid;
      if (w.team_units > 0) ok = ok && p.team_workers > 0 && p.team_run > 0;
      if (w.few_work > 0) ok = ok && p.few_workers > 0 && 4L * p.few_run * p.few_workers >= w.few_work;
      if (w.own_work > 0) ok = ok && p.own_workers > 0 && 4L * p.own_run * p.own_workers >= w.own_work;
      long slots = few_segments + 4L * p.few_workers;
      for (int k = 0; k < prefixes; ++k) {
        if (tiles[k] == 0) continue;
        const int span = p.team_aligned ? units[k] : hkv * units[k], cuts = (span + p.team_run - 1) / p.team_run;
        slots += (long)(p.team_aligned ? hkv * cuts : hkv + cuts) * wide[k];
      }
      ok = ok && slots <= wide_slots;
      if (w.own_work > 0) ok = ok && (long)hkv * rows - 1 + (w.own_work - 1) / p.own_run < own_slots;
      ++checked;
      if (!ok && bad++ < 5)
        std::printf("hkv %d G %d prefixes %d rows %d grid %d: workers %d %d %d, run %d aligned %d, slots %ld of %ld\n", hkv,
                    group, prefixes, rows, grid, p.team_workers, p.few_workers, p.own_workers, p.team_run, p.team_aligned,
                    slots, wide_slots);
    }
  }
  std::printf("%ld checked, %ld bad\n", checked, bad);
  return bad != 0 || checked < 100000;
}
