// The pick of csrc/select.hip on the host, by its keys and bins (csrc/key_bins.h): random rows of
// scores, with many infinite and undefined ones, in one chunk and in several, against a sort.
// -DWRAPPING: bins whose end is worked out without a look at what it may pass (the walk has to find it).
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <random>
#include <vector>

#include "key_bins.h"

namespace {

using Keys = std::vector<uint64_t>;
constexpr int kBins = 1024, kRanked = 64;

struct Bins : ekv::KeyBins {
  void enter(int bin, int shift) {
#ifdef WRAPPING
    from += (uint64_t)bin << shift;
    to = std::min(to, from + (uint64_t)((1ull << shift) - 1));
#else
    KeyBins::enter(bin, shift);
#endif
  }
};

struct Last {
  uint64_t key;
  int ties;
};

// The last of the `need` largest among few keys (0: none), and how many equal to it are taken.
Last rank(Keys keys, int need) {
  std::sort(keys.begin(), keys.end(), std::greater<uint64_t>());
  const uint64_t last = keys[need - 1];
  const int above = (int)(std::lower_bound(keys.begin(), keys.end(), last, std::greater<uint64_t>()) - keys.begin());
  return {last, need - above};
}

// Picker::find_last, one key after the other.
Last find_last(const Keys& keys, int need) {
  if ((int)keys.size() <= kRanked) return rank(keys, need);
  Bins in;
  in.from = ~0ull;
  in.to = 0;
  for (uint64_t k : keys) {
    if (k != 0) in.from = std::min(in.from, k);
    in.to = std::max(in.to, k);
  }
  while (in.from < in.to) {
    const int shift = in.shift();
    std::vector<int> bins(kBins);
    for (uint64_t k : keys)
      if (in.holds(k)) {
        if (in.bin(k, shift) >= (uint32_t)kBins) return {0, -1};
        ++bins[in.bin(k, shift)];
      }
    int bin = kBins - 1, over = 0;
    while (bin > 0 && over + bins[bin] < need) over += bins[bin--];
    need -= over;
    in.enter(bin, shift);
    if (need == bins[bin]) return {in.from - 1, 0};
    if (bins[bin] <= kRanked && in.from < in.to) {
      Keys few;
      for (uint64_t k : keys)
        if (in.holds(k)) few.push_back(k);
      if ((int)few.size() != bins[bin]) return {0, -1};
      return rank(few, need);
    }
  }
  return {in.from, need};
}

// Picker::list_above: the places' keys, of at most `room` places (-1 behind them: more were taken).
std::vector<int> list_above(const Keys& keys, Last last, int room) {
  std::vector<int> out;
  int seen = 0;
  for (int i = 0; i < (int)keys.size(); ++i)
    if (keys[i] > last.key || (keys[i] == last.key && seen++ < last.ties)) {
      if ((int)out.size() == room) return out.push_back(-1), out;
      out.push_back(i);
    }
  return out;
}

// The `need` largest of a row in chunks that keep their best, and a join of what they kept.
std::vector<int> pick(const Keys& row, int chunk, int need) {
  const int n = (int)row.size();
  if (chunk >= n) return list_above(row, n > need ? find_last(row, need) : Last{0, 0}, need);
  const int kept = std::min(chunk, need), chunks = (n + chunk - 1) / chunk;
  Keys keys(chunks * kept, 0);
  std::vector<int> blocks(chunks * kept, -1);
  for (int c = 0; c < chunks; ++c) {
    const Keys part(row.begin() + c * chunk, row.begin() + std::min(n, (c + 1) * chunk));
    const auto best = list_above(part, (int)part.size() > need ? find_last(part, need) : Last{0, 0}, kept);
    for (int i = 0; i < (int)best.size(); ++i) {
      if (best[i] < 0) return best;
      keys[c * kept + i] = part[best[i]];
      blocks[c * kept + i] = c * chunk + best[i];
    }
  }
  auto out = list_above(keys, find_last(keys, need), need);
  for (int& i : out) i = i < 0 ? -1 : blocks[i];
  return out;
}

}  // namespace

int main() {
  std::mt19937_64 random(1);
  auto below = [&](int n) { return (int)(random() % (uint64_t)n); };
  const double inf = INFINITY, nan = NAN;
  int bad = 0, cases = 0;
  for (; cases < 20000; ++cases) {
    const int n = 2 + below(cases % 4 ? 400 : 3000), need = 1 + below(n - 1);
    std::vector<double> scores(n);
    // a share of each kind, and finite scores of either sign or both, over few or many powers of two, some of them equal
    const int share_nan = below(3) ? below(60) : 0, share_up = below(3) ? below(60) : 0, share_down = below(3) ? below(60) : 0;
    const int sign = below(3), powers = below(2) ? 2 : 500, kinds = below(3) ? 1 << 30 : 1 + below(4);
    for (double& x : scores) {
      const int k = below(100);
      const int64_t grain = (int64_t)(random() % (uint64_t)kinds);
      x = std::ldexp(1.0 + (double)grain / (1 << 30), below(powers) - powers / 2);
      if (sign == 0 || (sign == 1 && below(2))) x = -x;
      if (k < share_nan) x = nan;
      else if (k < share_nan + share_up) x = inf;
      else if (k < share_nan + share_up + share_down) x = -inf;
      else if (below(50) == 0) x = below(2) ? 0.0 : -0.0;
    }
    Keys row(n);
    for (int i = 0; i < n; ++i) row[i] = ekv::score_key(scores[i]);
    std::vector<int> want(n);
    for (int i = 0; i < n; ++i) want[i] = i;
    std::stable_sort(want.begin(), want.end(), [&](int a, int b) {
      const double x = scores[a], y = scores[b];
      return x != x ? y == y : (y == y && x > y);
    });
    want.resize(need);
    std::sort(want.begin(), want.end());
    for (int chunk : {n, 64, 256}) {
      if (chunk < n && (n + chunk - 1) / chunk * std::min(chunk, need) <= need) continue;   // (a join picks among more)
      if (pick(row, chunk, need) == want) continue;
      if (bad++ < 5) std::printf("case %d: %d of %d in chunks of %d (%d%% NaN, %d%% inf, %d%% -inf)\n", cases, need, n, chunk, share_nan, share_up, share_down);
    }
  }
  std::printf("%d bad of %d\n", bad, cases);
  return bad != 0;
}
