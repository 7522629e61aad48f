// Every launch's pieces, worker by worker, against what the merge is told: each unit of
// each column once, every piece in a slot of its own inside the workspace, and the merge
// reads exactly the pieces of its columns.
#include <cstdio>
#include <map>
#include <random>

#include "model.h"

using namespace ekv;

namespace {

struct Made {           // what lies in a slot: units [u0, u1) of this segment, columns from `column` of its kind
  int kind, row, kvh, column, u0, u1;
};

const char* check(const Launch& l) {
  std::map<int, Made> wide, own;   // by slot
  // streams: a wave takes an equal run of the flat space of its kind
  auto stream = [&](std::map<int, Made>& to, int kind, int row, int kvh, int begin, int units, int slot, int run, int workers) -> const char* {
    int u = 0;
    while (u < units) {   // units begin + 1 ..: the segment's start is at `begin`
      const int w = (begin + 1 + u) / run, end = std::min(units, (w + 1) * run - begin - 1);
      if (w >= workers) return "a unit that no worker takes";
      if (!to.emplace(stream_slot(slot, kvh, w), Made{kind, row, kvh, 0, u, end}).second) return "two pieces in one slot";
      u = end;
    }
    return nullptr;
  };
  int flat = 0;
  std::vector<int> own_base(l.own.size());
  for (size_t s = 0; s < l.own.size(); ++s) {
    const int units = Launch::units_of(l.own[s]);
    own_base[s] = flat;
    if (units == 0) continue;
    for (int h = 0; h < l.hkv; ++h, flat += units + 1)
      if (const char* e = stream(own, kNone, (int)s, h, flat, units, own_slot0((int)s, l.hkv), l.plan.own_run, 4 * l.plan.own_workers)) return e;
  }
  for (size_t p = 0; p < l.prefix.size(); ++p) {
    if (l.split[p].rest > 0)
      for (int h = 0; h < l.hkv; ++h)
        if (const char* e = stream(wide, kFew, (int)p, h, l.base[kFew][p] + h * (l.units[p] + 1), l.units[p], l.slot[kFew][p],
                                   l.plan.few_run, 4 * l.plan.few_workers))
          return e;
    if (l.split[p].tiles == 0) continue;
    const Teams t(l.plan, l.units[p], l.hkv);
    for (int work = 0; work < l.of_kind[kTeam][p]; ++work) {
      const int team = work / l.split[p].tiles, tile = work % l.split[p].tiles, k = team / t.cuts;
      const int from = k * t.span + (team - k * t.cuts) * t.run, to = std::min((k + 1) * t.span, from + t.run);
      if (from >= to) return "a team without units";
      for (int u = from; u < to;) {
        const int h = u / l.units[p], u0 = u - h * l.units[p], u1 = std::min(l.units[p], u0 + to - u);
        const int first = tile_slot(l.plan, l.team_slot0 + l.slot[kTeam][p], l.split[p].wide, team, h, tile);
        for (int w = 0; w < 4; ++w) {
          if (128 * tile + 32 * w >= l.count[p] * l.group - l.split[p].rest) break;   // (a wave without columns)
          if (!wide.emplace(first + w, Made{kTeam, (int)p, h, 128 * tile + 32 * w, u0, u1}).second) return "two pieces in one slot";
        }
        u += u1 - u0;
      }
    }
  }
  if (!wide.empty() && (wide.begin()->first < 0 || wide.rbegin()->first >= l.size.wide_slots)) return "a wide slot outside the workspace";
  if (!own.empty() && (own.begin()->first < 0 || own.rbegin()->first >= l.size.own_slots)) return "an own slot outside the workspace";

  // the merge: a few sequences of every prefix (its first, its last, the ends of its tiles), every KV head
  for (size_t s = 0; s < l.own.size(); ++s) {
    Describe d{int4{0, 0, 0, 0}, int4{0, 0, 1, 0}, int4{0, 0, 0, 0}};
    int first = l.before, kind = kNone, j = 0, p = -1;
    for (size_t i = 0; i < l.prefix.size(); first += l.count[i++]) {
      if ((int)s < first || (int)s >= first + l.count[i] || l.prefix[i] <= 0) continue;
      const int column = ((int)s - first) * l.group, tiled = l.count[i] * l.group - l.split[i].rest;
      p = (int)i;
      kind = column < tiled ? kTeam : kFew;
      j = column < tiled ? column : column - tiled;
      describe_columns(d, l.plan, kind, l.hkv, l.units[i], l.split[i].wide, l.base[kind][i],
                       (kind == kTeam ? l.team_slot0 : 0) + l.slot[kind][i], j);
    }
    const int units = Launch::units_of(l.own[s]);
    if (units > 0) d.own = int4{own_base[s] + 1, units, l.plan.own_run, 0};
    for (int h = 0; h < l.hkv; ++h) {
      const PieceSlots w = prefix_pieces(d, h), o = own_pieces(d, (int)s, l.hkv, h);
      int next = 0;
      for (int k = 0; k < w.n; ++k) {
        const auto it = wide.find(w.slot + k * w.step);
        if (it == wide.end()) return "the merge reads a slot that nobody writes";
        const Made& m = it->second;
        if (m.kind != kind || m.row != p || m.kvh != h || m.u0 != next) return "the merge reads another piece";
        if (m.column + d.slots.w != j || d.slots.w + l.group > 32) return "the merge reads other columns";
        next = m.u1;
      }
      if (next != (p >= 0 ? l.units[p] : 0)) return "units of a prefix that the merge does not read";
      next = 0;
      for (int k = 0; k < o.n; ++k) {
        const auto it = own.find(o.slot + k * o.step);
        if (it == own.end()) return "the merge reads an own slot that nobody writes";
        const Made& m = it->second;
        if (m.row != (int)s || m.kvh != h || m.u0 != next) return "the merge reads another own piece";
        next = m.u1;
      }
      if (next != units) return "own units that the merge does not read";
    }
  }
  return nullptr;
}

}  // namespace

int main() {
  std::mt19937 rng(1);
  auto in = [&](int lo, int hi) { return (int)(lo + rng() % (unsigned)(hi - lo + 1)); };
  long checked = 0, aligned = 0, rounds = 0, crossed = 0;
  for (int it = 0; it < 12000; ++it) {
    Launch l;
    l.hkv = in(1, 12);
    l.group = 1 << in(0, 4);
    l.bytes8 = in(0, 1);
    l.resident = in(0, 1) ? kMaxSharedGrid : in(1, kMaxSharedGrid);
    const int prefixes = in(0, 3) ? in(0, 4) : in(1, 90);
    int longest = 1, own = in(0, 12) ? 1 << in(0, 11) : 0, blocks_s = 1;
    l.before = in(0, 3) ? 0 : in(0, 5);
    int rows = l.before + in(0, 3);
    for (int p = 0; p < prefixes; ++p) {
      l.count.push_back(in(0, 4) ? in(0, 1 << in(0, 8)) : 0);
      l.prefix.push_back(in(0, 8) ? in(1, 1 << in(1, 15)) : 0);
      rows += l.count[p];
      longest = std::max(longest, l.prefix[p]);
    }
    for (int s = 0; s < rows; ++s) l.own.push_back(in(0, 3) ? in(0, own) : 0);
    for (int n : l.own) blocks_s = std::max(blocks_s, (n + 15) / 16);
    if (rows == 0 || (long)l.hkv * rows > 3000 || !l.make((longest + in(0, 64) + 15) / 16, blocks_s + in(0, 8))) continue;
    if (const char* wrong = check(l)) {
      std::printf("%s: hkv %d G %d prefixes %d rows %d grid %d workers %d %d %d run %d aligned %d\n", wrong, l.hkv, l.group, prefixes, rows,
                  l.grid, l.plan.team_workers, l.plan.few_workers, l.plan.own_workers, l.plan.team_run, l.plan.team_aligned);
      return 1;
    }
    ++checked;
    aligned += l.plan.team_aligned;
    rounds += l.team_total > l.plan.team_workers;
    crossed += !l.plan.team_aligned && l.work.team_units > 0;
  }
  std::printf("%ld checked: teams in one segment %ld, across segments %ld, in rounds %ld\n", checked, aligned, crossed, rounds);
  return checked < 5000 || aligned < 500 || crossed < 500 || rounds < 100;
}
