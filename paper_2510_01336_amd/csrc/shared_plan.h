// Attention of a call whose sequences share pages, cut into pieces of work (host code only).
//
// The block tables of the call's sequences form a trie: a run of pages that the tables of several sequences begin with alike is a
// segment of all of them, the rest of a table a segment of its sequence alone.  A segment's query rows -- (row, query head of the KV head's
// group) of all its sequences, packed one after the other into tiles of sixteen -- meet its pages together, so that a page is
// read once for all of them.  Only pages that lie whole in front of every row of a sequence are taken as shared: those need no mask.
// Segments are cut into items of up to `block` tiles and a run of pages; a row's results over its items are joined at the end.
#pragma once
#include <algorithm>
#include <climits>
#include <functional>
#include <vector>

struct SharedSeq {            // one sequence of the call (m == 0: not taking part)
  int m = 0, p0 = 0;          // rows, position of the first
  int row0 = 0, qt0 = 0;      // its first row and q-tile in the call
  int n_pages = 0;            // pages up to the end of its last row (at the last step of a sequential pass)
  const int* pages = nullptr;
};
struct SharedItem {           // device layout: eight ints
  int tile0, n_tiles;         // packed tiles
  int seq, page0, page1;      // pages page0 .. page1-1 of that sequence's block table
  int slot0;                  // where its partial results go: slot of the first tile; -1: they are final
  int own;                    // 1: the sequence's own pages: masked by position, page1 cut at the end of the step's last row
  int pad;
};
struct SharedRow { int row, head, qpos, pos; };        // row of the call (-1: none), query head of the group, 16 * q-tile + row in it, position at step 0
struct SharedJoin { int row, head, first, count; };    // a row whose partials are entries first .. first+count-1
struct SharedPlan {
  std::vector<SharedItem> items;
  std::vector<SharedRow> rows;       // 16 per packed tile
  std::vector<SharedJoin> joins;
  std::vector<int> entries;          // 16 * slot + row in the tile
  int slots = 0;
  long pages_read = 0, pages_named = 0;   // by all items of a KV head; by the sequences one by one
  bool shares = false;
};

struct SharedSegment { std::vector<int> seqs; int page0, page1; bool own; };
// n pages in items of about `per`: how many items of how many pages (the last may have fewer)
struct SharedCuts { int cuts, run; };
inline SharedCuts shared_cuts(int n, int per) {
  const int c = std::max(1, (n + per - 1) / per), run = (n + c - 1) / c;
  return {(n + run - 1) / run, run};
}

// segments of the sequences `set`, whose tables are equal up to page `depth`, from there on
inline void shared_segments(const std::vector<SharedSeq>& q, const std::vector<int>& set, int depth, int least, std::vector<SharedSegment>& out) {
  std::vector<int> rest = set;
  auto shareable = [&](int b) { return std::min(q[b].p0 / 64, q[b].n_pages); };
  while (!rest.empty()) {
    const int b0 = rest[0];
    std::vector<int> same, other;
    for (int b : rest) {
      const bool joins = b == b0 || (depth < shareable(b) && depth < shareable(b0) && q[b].pages[depth] == q[b0].pages[depth]);
      (joins ? same : other).push_back(b);
    }
    rest.swap(other);
    int end = depth;
    if (same.size() > 1) {
      auto alike = [&](int p) {
        for (int b : same)
          if (p >= shareable(b) || q[b].pages[p] != q[b0].pages[p]) return false;
        return true;
      };
      while (alike(end)) ++end;
    }
    if (same.size() == 1) {
      out.push_back({same, depth, q[b0].n_pages, true});
    } else if (end - depth < least) {       // too short to be worth a segment: each reads it by itself
      std::vector<SharedSegment> below;
      shared_segments(q, same, end, least, below);
      for (SharedSegment& s : below) {
        if (s.page0 == end) s.page0 = depth;
        out.push_back(s);
      }
    } else {
      out.push_back({same, depth, end, false});
      shared_segments(q, same, end, least, out);
    }
  }
}

// Cost of an item in microseconds on its half of a compute unit: fitted to 484 timings (eleven batches of 2 to 64 sequences, each cut in 44 ways;
// the cuts that the fit chooses take 1.03 of the quickest ones' time in the mean, 1.09 at the worst).  Of one or two tiles, four or two pages
// go at a time; of more, every page costs its way through LDS and its tiles' products, 1.13 times that where
// the other half of every unit has such an item too (both: 0 with no unit shared so, 1 with all).
inline double shared_item_us(int tiles, int pages, double both) {
  if (tiles <= 2) return 1.7 * (tiles == 1 ? (pages + 3) / 4 : (pages + 1) / 2);
  return pages * (0.77 + 0.125 * tiles) * (1 + 0.13 * both);
}
constexpr double kSharedSlotUs = 0.034;               // a tile's partial results written, read and joined
constexpr double kSharedPageUs = 2.7;                 // a page of every KV head read from memory: this by the places that run at a time

// rep: query heads per KV head; most_slots: room for partial results; wgs: items of one KV head that run at a time; least: pages of
// a shared segment at the least; share: false keeps every sequence to itself; per_forced > 0: pages per item.
inline SharedPlan plan_shared(const std::vector<SharedSeq>& q, int rep, int most_slots, int wgs, int least, bool share, int per_forced = 0) {
  const int block = 8;
  SharedPlan P;
  std::vector<int> set;
  for (int b = 0; b < (int)q.size(); ++b)
    if (q[b].m > 0) { set.push_back(b); P.pages_named += q[b].n_pages; }
  std::vector<SharedSegment> segs;
  if (share) shared_segments(q, set, 0, least, segs);
  else for (int b : set) segs.push_back({{b}, 0, q[b].n_pages, true});
  // packed rows
  struct Placed { int tile0, tiles; };
  std::vector<Placed> at;
  int n_rows = 0;
  for (int b : set) n_rows = std::max(n_rows, q[b].row0 + q[b].m);
  std::vector<int> parts((size_t)n_rows * rep, 0);     // segments of every (row, head)
  for (const SharedSegment& s : segs) {
    const int tile0 = (int)P.rows.size() / 16;
    for (int b : s.seqs)
      for (int i = 0; i < q[b].m; ++i)
        for (int h = 0; h < rep; ++h) {
          P.rows.push_back({q[b].row0 + i, h, q[b].qt0 * 16 + i * rep + h, q[b].p0 + i});
          parts[(size_t)(q[b].row0 + i) * rep + h]++;
        }
    while (P.rows.size() % 16) P.rows.push_back({-1, 0, q[s.seqs[0]].qt0 * 16, -1});
    at.push_back({tile0, (int)P.rows.size() / 16 - tile0});
    P.shares |= s.seqs.size() > 1;
    P.pages_read += (long)(s.page1 - s.page0) * ((at.back().tiles + block - 1) / block);
  }
  // Pages per item, of shared segments and of the sequences' own: the pair whose items, dealt in their order to whichever of `wgs` places is free first,
  // are done soonest, the joining of the partial results counted in.
  int longest[2] = {1, 1};                              // shared, own
  for (const SharedSegment& s : segs) longest[s.own] = std::max(longest[s.own], s.page1 - s.page0);
  std::vector<double> free_at;
  long distinct = 0;
  for (const SharedSegment& s : segs) distinct += s.page1 - s.page0;
  auto schedule = [&](const int* per, double& us) {
    long slots = 0, wide = 0;
    for (size_t i = 0; i < segs.size(); ++i)
      wide += (long)shared_cuts(segs[i].page1 - segs[i].page0, per[segs[i].own]).cuts * ((at[i].tiles + block / 2 - 1) / block);
    const double both = std::min(1.0, std::max(0.0, 2.0 * wide / wgs - 1));
    free_at.assign(wgs, 0.0);
    double end = 0;
    for (int own = 0; own < 2; ++own)
      for (size_t i = 0; i < segs.size(); ++i) {
        if (segs[i].own != (own == 1)) continue;
        const int n = segs[i].page1 - segs[i].page0;
        const auto [cuts, run] = shared_cuts(n, per[own]);
        slots += (long)at[i].tiles * cuts;
        for (int c = 0; c < cuts; ++c)
          for (int t = 0; t < at[i].tiles; t += block) {
            std::pop_heap(free_at.begin(), free_at.end(), std::greater<double>());
            double& f = free_at.back();
            f += shared_item_us(std::min(block, at[i].tiles - t), std::min(run, n - c * run), both);
            end = std::max(end, f);
            std::push_heap(free_at.begin(), free_at.end(), std::greater<double>());
          }
      }
    us = std::max(end, kSharedPageUs * distinct / wgs) + kSharedSlotUs * slots;
    return slots <= most_slots;
  };
  int per[2] = {longest[0], longest[1]};
  if (per_forced > 0) {
    double us = 0;
    per[0] = per[1] = per_forced;
    while ((per[0] < longest[0] || per[1] < longest[1]) && !schedule(per, us)) { per[0]++; per[1]++; }
  } else {
    double best = 1e30;
    auto tries = [](int n, int most) {                  // numbers of items of the longest segment, finer where they are few
      std::vector<int> c;
      for (int k = 1; k <= std::min(n, most); k += 1 + k / 6) c.push_back((n + k - 1) / k);
      return c;
    };
    for (int own : tries(longest[1], 8))
      for (int joint : P.shares ? tries(longest[0], wgs) : std::vector<int>{1}) {
        const int p[2] = {joint, own};
        double us = 0;
        if (schedule(p, us) && us < best) { best = us; per[0] = joint; per[1] = own; }
      }
  }
  // items: the cuts of a segment one after the other, all its blocks of a cut together, so that workgroups that run at the same time read the same pages
  std::vector<int> slot_of;                             // per segment: first slot
  std::vector<int> cuts_of(segs.size());
  for (size_t i = 0; i < segs.size(); ++i) {
    cuts_of[i] = shared_cuts(segs[i].page1 - segs[i].page0, per[segs[i].own]).cuts;
    bool final = cuts_of[i] == 1;
    for (int r = at[i].tile0 * 16; final && r < (at[i].tile0 + at[i].tiles) * 16; ++r)
      final = P.rows[r].row < 0 || parts[(size_t)P.rows[r].row * rep + P.rows[r].head] == 1;
    slot_of.push_back(final ? -1 : P.slots);
    if (!final) P.slots += cuts_of[i] * at[i].tiles;
  }
  for (int pass = 0; pass < 2; ++pass)                  // shared segments first: their items are the long ones
    for (size_t i = 0; i < segs.size(); ++i) {
      if (segs[i].own != (pass == 1)) continue;
      const auto [cuts, run] = shared_cuts(segs[i].page1 - segs[i].page0, per[segs[i].own]);
      for (int c = 0; c < cuts; ++c)
        for (int t = 0; t < at[i].tiles; t += block)
          P.items.push_back({at[i].tile0 + t, std::min(block, at[i].tiles - t), segs[i].seqs[0], segs[i].page0 + c * run,
                             std::min(segs[i].page1, segs[i].page0 + (c + 1) * run), slot_of[i] < 0 ? -1 : slot_of[i] + c * at[i].tiles + t,
                             segs[i].own ? 1 : 0, 0});
    }
  // joins
  std::vector<std::vector<int>> of((size_t)n_rows * rep);
  for (size_t i = 0; i < segs.size(); ++i) {
    if (slot_of[i] < 0) continue;
    for (int t = 0; t < at[i].tiles; ++t)
      for (int r = 0; r < 16; ++r) {
        const SharedRow& w = P.rows[(size_t)(at[i].tile0 + t) * 16 + r];
        if (w.row < 0) continue;
        for (int c = 0; c < cuts_of[i]; ++c) of[(size_t)w.row * rep + w.head].push_back((slot_of[i] + c * at[i].tiles + t) * 16 + r);
      }
  }
  for (int r = 0; r < n_rows * rep; ++r) {
    if (of[r].empty()) continue;
    P.joins.push_back({r / rep, r % rep, (int)P.entries.size(), (int)of[r].size()});
    P.entries.insert(P.entries.end(), of[r].begin(), of[r].end());
  }
  return P;
}

// Whether a call of a session takes the plan instead of reading every sequence's pages by itself.
inline bool shared_pays(const SharedPlan& P) { return P.shares && 2 * P.pages_read <= P.pages_named; }
