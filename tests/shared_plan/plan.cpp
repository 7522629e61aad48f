// Prints how one launch is divided.  Standard input: hkv group bytes8 blocks_p blocks_s
// before, then the number of prefixes and each one's sequences and tokens, then the
// number of sequences and each one's tokens.
#include <cstdio>

#include "model.h"

int main() {
  Launch l;
  int bytes8 = 0, blocks_p = 0, blocks_s = 0, n = 0;
  if (std::scanf("%d %d %d %d %d %d %d", &l.hkv, &l.group, &bytes8, &blocks_p, &blocks_s, &l.before, &n) != 7) return 2;
  l.bytes8 = bytes8 != 0;
  for (int i = 0; i < n; ++i) {
    int count = 0, len = 0;
    if (std::scanf("%d %d", &count, &len) != 2) return 2;
    l.count.push_back(count);
    l.prefix.push_back(len);
  }
  if (std::scanf("%d", &n) != 1) return 2;
  for (int i = 0, len = 0; i < n; ++i) {
    if (std::scanf("%d", &len) != 1) return 2;
    l.own.push_back(len);
  }
  if (!l.make(blocks_p, blocks_s)) return 1;
  std::printf("grid=%d team_workers=%d few_workers=%d own_workers=%d team_work=%d team_tiles=%d team_run=%d team_aligned=%d "
              "few_run=%d own_run=%d merge_ways=%d min_units=%d team_units=%d few_work=%d own_work=%d\n",
              l.grid, l.plan.team_workers, l.plan.few_workers, l.plan.own_workers, l.team_total, l.work.team_tiles, l.plan.team_run,
              l.plan.team_aligned, l.plan.few_run, l.plan.own_run, l.size.merge_ways, l.size.min_units, l.work.team_units,
              l.work.few_work, l.work.own_work);
  return 0;
}
