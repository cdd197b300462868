// Host-side check of how the work of amk_attention_weights is divided (amk_weights_units.h): for one call it replays the blocks' runs and
// verifies that
//   * a sequence of impossible length has no units and no steps,
//   * every step of every unit of the other sequences is some block's, and only one's,
//   * a unit's steps are the query tiles from the first one on that sees one of its positions, up to the last.
// Usage: weights_units_check span nkv rows slots tokens blocks len...  -> prints "ok" or a diagnostic.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <tuple>
#include <vector>

#include "amk_weights_units.h"
using namespace amk;

template <int SPAN>
int check(const WeightsWork& p, int blocks) {
  std::vector<long long> steps(p.n_seqs);
  long long total = 0;
  for (int s = 0; s < p.n_seqs; s++) {
    const long long len = p.lens[s];
    const bool legal = len >= 0 && len + p.rows <= p.slots;
    const int n = weights_steps<SPAN>(p, p.lens[s]);
    if (!legal && (weights_units<SPAN>(p, p.lens[s]) || n)) { printf("length %lld: %d steps\n", len, n); return 1; }
    long long want = 0;
    if (legal)
      for (long long key = 0; key < len + p.rows; key += SPAN) {
        int first = 0;
        while (SPAN != kFewSpan && first < p.q_tiles && len + (long long)(first + 1) * p.tokens - 1 < key) first++;
        if (first_q_tile<SPAN>(p, p.lens[s], (int)(key / SPAN)) != first) { printf("length %lld: first tile of the unit at %lld\n", len, key); return 1; }
        want += SPAN == kFewSpan ? 1 : p.q_tiles - first;
      }
    if (n != want) { printf("length %lld: %d steps, not %lld\n", len, n, want); return 1; }
    steps[s] = (long long)n * p.nkv, total += steps[s];
  }
  const long long per = (total + blocks - 1) / blocks;
  std::map<std::tuple<int, int, int, int>, int> seen;
  for (int b = 0; b < blocks && b * per < total; b++) {
    long long at = b * per;
    int s = 0;
    while (at >= steps[s]) at -= steps[s++];
    const int of_head = (int)(steps[s] / p.nkv), head = (int)(at / of_head);
    int unit, step;
    weights_place<SPAN>(p, p.lens[s], (int)(at - (long long)head * of_head), unit, step);
    const int start[6] = {s, head, unit, step, (int)(total - b * per < per ? total - b * per : per), p.lens[s]};
    WeightsWalk<SPAN> walk;
    walk.init(p, start);
    WeightsUnit u;
    while (walk.next(p, u)) {
      if (u.seq >= p.n_seqs || u.head >= p.nkv || u.begin < 0 || u.begin >= u.end || u.end > u.all) { printf("block %d: unit out of range\n", b); return 1; }
      for (int i = u.begin; i < u.end; i++) seen[{u.seq, u.head, u.at, u.first + i}]++;
    }
  }
  if ((long long)seen.size() != total) { printf("%zu steps worked on, not %lld\n", seen.size(), total); return 1; }
  for (const auto& x : seen)
    if (x.second != 1) { printf("a step worked on %d times\n", x.second); return 1; }
  printf("ok\n");
  return 0;
}

int main(int argc, char** argv) {
  if (argc < 8) return 2;
  std::vector<int> lens;
  for (int i = 7; i < argc; i++) lens.push_back(atoi(argv[i]));
  WeightsWork p{};
  p.lens = lens.data(), p.n_seqs = (int)lens.size();
  p.nkv = atoi(argv[2]), p.rows = atoi(argv[3]), p.slots = atoi(argv[4]), p.tokens = atoi(argv[5]);
  p.q_tiles = (p.rows + p.tokens - 1) / p.tokens;
  const int span = atoi(argv[1]), blocks = atoi(argv[6]);
  return span == kFewSpan ? check<kFewSpan>(p, blocks) : span == kManySpan ? check<kManySpan>(p, blocks) : 2;
}
