// A launch of shared-prefix decode on the host: what the entry point sizes, what the
// kernel counts and how it is divided, from the functions that both use.
#pragma once

#include <algorithm>
#include <vector>

#include "shared_plan.h"

struct Launch {
  // the call
  int hkv = 1, group = 1, resident = ekv::kMaxSharedGrid;
  bool bytes8 = false;
  std::vector<int> count, prefix;   // sequences and tokens of each prefix (in order, from sequence `before` on)
  std::vector<int> own;             // tokens of every sequence
  int before = 0;
  // what follows
  ekv::SharedSize size{};
  ekv::SharedWork work{};
  ekv::SharedPlan plan{};
  int grid = 0, few_segments = 0, team_slot0 = 0;
  std::vector<ekv::ColumnSplit> split;
  std::vector<int> units, base[3], slot[3], of_kind[3];   // by kind: where a prefix's work and slots begin, its work
  int few_total = 0, team_total = 0;

  static int units_of(int len) { return (len + 31) / 32; }

  // blocks: of the longest prefix and sequence that the batches state
  bool make(int blocks_p, int blocks_s) {
    using namespace ekv;
    if (!size_shared((int64_t)prefix.size(), (int64_t)own.size(), (blocks_p + 1) / 2, (blocks_s + 1) / 2, hkv, group, &size)) return false;
    grid = std::max(4, std::min(size.grid, resident));
    if ((int64_t)own.size() > 64 * grid) return false;
    work = SharedWork{};
    for (int n : own) work.own_work += n > 0 ? hkv * (units_of(n) + 1) : 0;
    few_segments = 0;
    split.clear();
    units.clear();
    for (size_t p = 0; p < prefix.size(); ++p) {
      const int n = prefix[p] > 0 ? count[p] : 0;
      split.push_back(ColumnSplit(n * group));
      units.push_back(n > 0 ? units_of(prefix[p]) : 0);
      if (split[p].rest > 0) {
        work.few_work += hkv * (units[p] + 1);
        few_segments += hkv;
      }
      work.team_tiles += split[p].tiles;
      work.team_units += hkv * split[p].tiles * units[p];
    }
    work.team_segments = hkv * work.team_tiles;
    plan = divide_work(work, grid, size.min_units, bytes8);
    team_slot0 = first_team_slot(plan, few_segments);
    for (int kind : {kFew, kTeam}) {
      int at = 0, slots = 0;
      base[kind].assign(prefix.size(), 0);
      slot[kind].assign(prefix.size(), 0);
      of_kind[kind].assign(prefix.size(), 0);
      for (size_t p = 0; p < prefix.size(); ++p) {
        const Amounts n(split[p], units[p], plan, kind, hkv);
        base[kind][p] = at;
        slot[kind][p] = slots;
        if (kind == kTeam ? split[p].tiles > 0 : split[p].rest > 0) {
          at += of_kind[kind][p] = n.work;
          slots += n.slots;
        }
      }
      (kind == kFew ? few_total : team_total) = at;
    }
    return true;
  }
};
