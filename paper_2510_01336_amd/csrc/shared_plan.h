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
  long pages_named = 0;              // by the sequences one by one
  bool shares = false;
  double us = 0;                          // estimated time on the device
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
  auto shareable = [&](int b) { return std::min(q[b].p0 / 64, q[b].n_pages); };
  std::vector<int> rest;                                // those that may share page `depth`, by that page
  for (int b : set) {
    if (depth < shareable(b)) rest.push_back(b);
    else out.push_back({{b}, depth, q[b].n_pages, true});
  }
  std::stable_sort(rest.begin(), rest.end(), [&](int x, int y) { return q[x].pages[depth] < q[y].pages[depth]; });
  for (size_t i = 0, j; i < rest.size(); i = j) {
    const int b0 = rest[i];
    for (j = i + 1; j < rest.size() && q[rest[j]].pages[depth] == q[b0].pages[depth]; ) ++j;
    if (j - i == 1) { out.push_back({{b0}, depth, q[b0].n_pages, true}); continue; }
    const std::vector<int> same(rest.begin() + i, rest.begin() + j);
    int end = depth + 1;
    auto alike = [&](int p) {
      for (int b : same)
        if (p >= shareable(b) || q[b].pages[p] != q[b0].pages[p]) return false;
      return true;
    };
    while (alike(end)) ++end;
    if (end - depth < least) {                          // too short to be worth a segment: each reads it by itself
      std::vector<SharedSegment> below;
      shared_segments(q, same, end, least, below);
      for (SharedSegment& s : below) {
        if (s.page0 == end) s.page0 = depth;
        out.push_back(std::move(s));
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
constexpr double kSharedJoinUs = 3.5;                 // the launch that joins them
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
  // shared segments first, then the sequences' own, the longer ones first: what takes longest is begun first
  std::stable_sort(segs.begin(), segs.end(), [](const SharedSegment& x, const SharedSegment& y) {
    return x.own != y.own ? y.own : x.page1 - x.page0 > y.page1 - y.page0;
  });
  // packed rows
  struct Placed { int tile0, tiles; };
  std::vector<Placed> at;
  int n_rows = 0;
  for (int b : set) n_rows = std::max(n_rows, q[b].row0 + q[b].m);
  std::vector<int> parts((size_t)n_rows * rep, 0);     // segments of every (row, head)
  P.rows.reserve(((size_t)n_rows * rep + 15) / 16 * 32 + 16 * segs.size());
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
  }
  // Pages per item, of shared segments and of the sequences' own: the pair whose items, dealt in their order to whichever of `wgs` places is free first,
  // are done soonest, the joining of the partial results counted in.  Segments alike are dealt together, and a pair is only dealt if the
  // work over all places and the longest item leave it a chance: the whole choice takes some microseconds of the host.
  int longest[2] = {1, 1};                              // shared, own
  struct Alike { int tiles, pages, own, alone, n; };      // alone: its rows have no other segment, so that uncut they need no joining
  std::vector<Alike> alike;
  long distinct = 0;
  for (size_t i = 0; i < segs.size(); ++i) {
    const int n = segs[i].page1 - segs[i].page0;
    longest[segs[i].own] = std::max(longest[segs[i].own], n);
    distinct += n;
    const Alike x = {at[i].tiles, n, segs[i].own, segs[i].page0 == 0 && segs[i].own, 1};
    if (!alike.empty() && alike.back().tiles == x.tiles && alike.back().pages == n && alike.back().own == x.own && alike.back().alone == x.alone) alike.back().n++;
    else alike.push_back(x);
  }
  std::vector<double> free_at;
  auto schedule = [&](const int* per, double best, double& us) {
    long slots = 0, wide = 0, items = 0;
    for (const Alike& s : alike) {
      const int cuts = shared_cuts(s.pages, per[s.own]).cuts;
      if (cuts > 1 || !s.alone) slots += (long)s.n * s.tiles * cuts;
      items += (long)s.n * cuts * ((s.tiles + block - 1) / block);
      wide += (long)s.n * cuts * ((s.tiles + block / 2 - 1) / block);
    }
    if (slots > most_slots) return false;
    const double both = std::min(1.0, std::max(0.0, 2.0 * wide / wgs - 1)), more = kSharedSlotUs * slots + (slots ? kSharedJoinUs : 0);
    auto each = [&](auto deal) {                        // runs of equal items, in their order
      for (const Alike& s : alike) {
        const auto [cuts, run] = shared_cuts(s.pages, per[s.own]);
        const int full = s.tiles / block, rest = s.tiles % block;
        if (full) { deal(shared_item_us(block, run, both), (long)s.n * full * (cuts - 1)); deal(shared_item_us(block, s.pages - (cuts - 1) * run, both), (long)s.n * full); }
        if (rest) { deal(shared_item_us(rest, run, both), (long)s.n * (cuts - 1)); deal(shared_item_us(rest, s.pages - (cuts - 1) * run, both), (long)s.n); }
      }
    };
    double all = 0, end = kSharedPageUs * distinct / wgs;
    each([&](double t, long n) { all += t * n; if (n) end = std::max(end, t); });
    end = std::max(end, all / wgs);
    if (end + more < best && items > wgs) {
      free_at.assign(wgs, 0.0);
      each([&](double t, long n) {
        for (; n > 0 && end + more < best; --n) {
          std::pop_heap(free_at.begin(), free_at.end(), std::greater<double>());
          end = std::max(end, free_at.back() += t);
          std::push_heap(free_at.begin(), free_at.end(), std::greater<double>());
        }
      });
    }
    us = end + more;
    return us < best;
  };
  int per[2] = {longest[0], longest[1]};
  P.us = 1e30;
  if (per_forced > 0) {
    per[0] = per[1] = per_forced;
    while ((per[0] < longest[0] || per[1] < longest[1]) && !schedule(per, 1e30, P.us)) { per[0]++; per[1]++; }
  } else {
    auto tries = [](int n, int most) {                  // numbers of items of the longest segment, finer where they are few
      std::vector<int> c;
      for (int k = 1; k <= std::min(n, most); k += 1 + k / 6) c.push_back((n + k - 1) / k);
      return c;
    };
    const std::vector<int> joint = P.shares ? tries(longest[0], wgs) : std::vector<int>{1};
    for (int own : tries(longest[1], 8))
      for (int j : joint) {
        const int p[2] = {j, own};
        double us = 0;
        if (schedule(p, P.us, us)) { P.us = us; per[0] = j; per[1] = own; }
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
  for (size_t i = 0; i < segs.size(); ++i) {
    const auto [cuts, run] = shared_cuts(segs[i].page1 - segs[i].page0, per[segs[i].own]);
    for (int c = 0; c < cuts; ++c)
      for (int t = 0; t < at[i].tiles; t += block)
        P.items.push_back({at[i].tile0 + t, std::min(block, at[i].tiles - t), segs[i].seqs[0], segs[i].page0 + c * run,
                           std::min(segs[i].page1, segs[i].page0 + (c + 1) * run), slot_of[i] < 0 ? -1 : slot_of[i] + c * at[i].tiles + t,
                           segs[i].own ? 1 : 0, 0});
  }
  // joins: every row's entries, counted, then placed
  std::vector<int> first((size_t)n_rows * rep, 0);
  auto each_entry = [&](auto f) {
    for (size_t i = 0; i < segs.size(); ++i)
      if (slot_of[i] >= 0)
        for (int r = 0; r < 16 * at[i].tiles; ++r) {
          const SharedRow& w = P.rows[(size_t)at[i].tile0 * 16 + r];
          if (w.row >= 0) f(w.row * rep + w.head, cuts_of[i], slot_of[i] * 16 + r, at[i].tiles * 16);
        }
  };
  each_entry([&](int r, int n, int, int) { first[r] += n; });
  int total = 0;
  for (int r = 0; r < n_rows * rep; ++r) {
    const int n = first[r];
    first[r] = total;
    if (n) P.joins.push_back({r / rep, r % rep, total, n});
    total += n;
  }
  P.entries.resize(total);
  each_entry([&](int r, int n, int e, int step) {
    for (int c = 0; c < n; ++c) P.entries[first[r]++] = e + c * step;
  });
  return P;
}

// Whether a call of a session takes the plan instead of reading every sequence's pages by itself, which takes the time of the pages that the
// sequences name, a page of every KV head 1.8 us by the places that run at a time (from the caches, 9.3 TB/s; shared ones lie there).  The
// plan's launches and waits cost 6 us more than theirs, the launch that joins among them.  Measured on calls of 14 layers, 8 KV heads, 114 batches of 2 to 48 sequences
// that share 128 to 8192 positions, 20 to 1500 of their own, 1 and 8 rows each, both forms: the rule takes the slower form of seven, 0.1 to 2.3 us a
// layer slower.  A whole call of 48 sequences that share 8192 positions takes 3220 us by sequences and 1220 by the plan (eight rows each:
// 4195 and 2703), of 16 that share 2048 630 and 662 (the largest loss), of 4 that share 256 616 and 703 with eight rows (left to the
// other form).  A plan for every batch that names twice the pages that it reads lost 150 us a layer over the 114.
inline bool shared_pays(long pages_named, int wgs, double plan_us) { return plan_us + 2.5 < 1.8 * pages_named / wgs; }
