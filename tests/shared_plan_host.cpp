// Checks of the work plan of attention over shared pages (csrc/shared_plan.h) on random block tables: prints "ok <plans>" or what is wrong.
#include "../paper_2510_01336_amd/csrc/shared_plan.h"
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>

#define CHECK(...) do { if (!(__VA_ARGS__)) { printf("failed: %s (plan %d, line %d)\n", #__VA_ARGS__, plan, __LINE__); return 1; } } while (0)

int main(int argc, char** argv) {
  const int plans = argc > 1 ? atoi(argv[1]) : 2000;
  std::mt19937 rng(7);
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  for (int plan = 0; plan < plans; ++plan) {
    const int B = pick(1, plan % 10 ? 12 : 70), rep = pick(1, 16), most_rows = pick(1, plan % 3 ? 4 : 20), steps = pick(1, 5);
    const int depth = pick(1, plan % 7 ? 30 : 300);
    std::vector<std::vector<int>> tables(B);
    std::vector<SharedSeq> q(B);
    int next = 0, row = 0, qt = 0;
    for (int b = 0; b < B; ++b) {
      // a table begins like that of an earlier sequence, up to a random page
      if (b && pick(0, 3)) {
        const std::vector<int>& from = tables[pick(0, b - 1)];
        tables[b].assign(from.begin(), from.begin() + pick(0, (int)from.size()));
      }
      const int taken = (int)tables[b].size(), more = pick(taken ? 0 : 1, std::max(1, depth - taken));
      for (int i = 0; i < more; ++i) tables[b].push_back(next++);
      const int room = (int)tables[b].size() * 64;
      const int m = pick(0, 4) ? std::min(pick(1, most_rows), room) : 0, add = std::min(steps - 1, room - m);
      if (!m) continue;
      q[b].m = m;
      q[b].p0 = pick(0, 2) ? room - m - add : pick(0, room - m - add);
      q[b].row0 = row; q[b].qt0 = qt;
      q[b].n_pages = (q[b].p0 + m + add + 63) / 64;
      q[b].pages = tables[b].data();
      row += m; qt += (m * rep + 15) / 16;
    }
    if (!row) continue;
    const int tiles = (row * rep + 15) / 16 + B, room = pick(0, 1) ? 64 * tiles : 12 * tiles, least = pick(1, 4);
    const bool share = pick(0, 4) != 0;
    const SharedPlan P = plan_shared(q, rep, room, pick(1, 64), least, share, pick(0, 3) ? 0 : pick(1, 20));
    CHECK(P.rows.size() % 16 == 0);
    if (!share) CHECK(!P.shares);
    std::set<int> used;
    std::map<std::pair<int, int>, std::vector<int>> pages;         // (row, head) -> pages met
    std::map<std::pair<int, int>, std::vector<int>> slots;         // ... and where its partials lie
    std::map<std::pair<int, int>, int> finals;
    std::vector<int> seq_of(row);
    for (int b = 0; b < B; ++b) for (int i = 0; i < q[b].m; ++i) seq_of[q[b].row0 + i] = b;
    for (const SharedItem& it : P.items) {
      CHECK(it.n_tiles >= 1 && it.n_tiles <= 8 && it.tile0 >= 0 && (size_t)(it.tile0 + it.n_tiles) * 16 <= P.rows.size());
      CHECK(it.seq >= 0 && it.seq < B && q[it.seq].m > 0);
      CHECK(it.page0 >= 0 && it.page0 < it.page1 && it.page1 <= q[it.seq].n_pages);
      CHECK(P.rows[it.tile0 * 16].row >= 0);
      int before = -1;
      for (int t = 0; t < it.n_tiles; ++t) {
        if (it.slot0 >= 0) { CHECK(it.slot0 + t < P.slots); CHECK(used.insert(it.slot0 + t).second); }
        for (int c = 0; c < 16; ++c) {
          const SharedRow& w = P.rows[(it.tile0 + t) * 16 + c];
          CHECK(w.qpos >= 0 && w.qpos < 16 * qt);
          if (w.row < 0) continue;
          CHECK(w.row < row && w.head >= 0 && w.head < rep);
          const int b = seq_of[w.row];
          CHECK(w.pos == q[b].p0 + w.row - q[b].row0 && w.qpos == q[b].qt0 * 16 + (w.row - q[b].row0) * rep + w.head);
          if (it.own) {
            CHECK(b == it.seq && w.pos >= before);                 // (the first row of an item sees the least)
            before = w.pos;
          } else {
            for (int g = it.page0; g < it.page1; ++g) CHECK(q[b].pages[g] == q[it.seq].pages[g]);
            CHECK(it.page1 * 64 <= q[b].p0);                       // whole pages in front of every row
          }
          for (int g = it.page0; g < it.page1; ++g) pages[{w.row, w.head}].push_back(g);
          if (it.slot0 >= 0) slots[{w.row, w.head}].push_back((it.slot0 + t) * 16 + c);
          else finals[{w.row, w.head}]++;
        }
      }
    }
    for (int r = 0; r < row; ++r)
      for (int h = 0; h < rep; ++h) {
        std::vector<int>& p = pages[{r, h}];
        std::sort(p.begin(), p.end());
        CHECK((int)p.size() == q[seq_of[r]].n_pages);
        for (size_t i = 0; i < p.size(); ++i) CHECK(p[i] == (int)i);
        CHECK(finals[{r, h}] <= 1 && (finals[{r, h}] == 1) == slots[{r, h}].empty());
      }
    std::set<std::pair<int, int>> joined;
    size_t at = 0;
    for (const SharedJoin& j : P.joins) {
      CHECK(joined.insert({j.row, j.head}).second && j.first == (int)at && j.count >= 1);
      std::vector<int> e(P.entries.begin() + j.first, P.entries.begin() + j.first + j.count), s = slots[{j.row, j.head}];
      std::sort(e.begin(), e.end()); std::sort(s.begin(), s.end());
      CHECK(e == s);
      at += j.count;
    }
    CHECK(at == P.entries.size());
    size_t with = 0;
    for (auto& s : slots) with += !s.second.empty();
    CHECK(with == joined.size());
    bool fits_uncut = true;
    if (!share && P.slots > room) fits_uncut = false;
    CHECK(fits_uncut);                                             // sequences by themselves always fit where a tile has a slot
  }
  printf("ok %d\n", plans);
  return 0;
}
