// Host plan of pie_fork_kvpage: plain C++, no HIP.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <vector>

struct PageMove { int32_t src, dst; };       // src -1: the page kept at the start of the run
struct PageRun { int32_t first, n, keep; };  // moves [first, first + n) in order; keep >= 0: a page read before them
#define FORK_MOVES 160  // moves (and runs) of a launch, which travel as kernel arguments (4 KiB at most)
#define FORK_FAN 16     // moves of a run where any order will do

// Moves dst[i] <- src[i] (all from the pages as they were; destinations distinct) as launches of independent runs of moves, in an
// order that needs no second buffer: a page is written after every move that reads it.  A page that is read is a hub, its moves stand
// together (the source is loaded once), and the hubs form trees (a hub's parent is the page it becomes) some of which hang on
// a cycle.  A tree is one run, deepest hubs first; a hub alone is cut into runs of FORK_FAN moves.  A cycle c0 <- c1 <- .. <- c0
// starts with keeping c0, and its last move stores what was kept.  Runs that do not fit a launch go on in the next; what a cycle
// keeps is put down meanwhile in the page that its next move overwrites, whose contents nobody needs any more.
struct ForkPlan {
  struct Launch { int32_t move0, n_moves, run0, n_runs; };  // (PageRun::first counts from move0)
  std::vector<PageMove> moves;
  std::vector<PageRun> runs;
  std::vector<Launch> launches;

  ForkPlan(const int32_t* src, const int32_t* dst, int n) {
    given.reserve(n);
    for (int i = 0; i < n; ++i)
      if (src[i] != dst[i]) given.push_back(PageMove{src[i], dst[i]});
    std::stable_sort(given.begin(), given.end(), [](const PageMove& a, const PageMove& b) { return a.src < b.src; });
    for (size_t i = 0; i < given.size(); ++i)
      if (i == 0 || given[i].src != given[i - 1].src) first.push_back((int32_t)i);
    const int n_hubs = (int)first.size();
    first.push_back((int32_t)given.size());
    parent.assign(n_hubs, -1);
    kids.resize(n_hubs);
    for (const PageMove& m : given) {
      const int h = hub_of(m.dst);
      if (h < 0) continue;
      parent[h] = hub_of(m.src);
      kids[parent[h]].push_back(h);
    }
    seen.assign(n_hubs, 0);
    for (int h = 0; h < n_hubs; ++h)
      if (parent[h] < 0) {
        begin(-1, kids[h].empty());
        tree(h, -1);
      }
    std::vector<char> walked(n_hubs, 0);
    std::vector<int32_t> cycle;
    for (int h = 0; h < n_hubs; ++h) {
      if (seen[h]) continue;
      int x = h;  // up from h until the cycle has been walked once: x is on it
      while (!walked[x]) { walked[x] = 1; x = parent[x]; }
      cycle.clear();
      for (int y = x;;) {
        cycle.push_back(y);
        y = parent[y];
        if (y == x) break;
      }
      const int L = (int)cycle.size();
      for (int y : cycle) seen[y] = 1;
      begin(page(cycle[0]), false);
      for (int y : cycle)
        for (int k : kids[y])
          if (!seen[k]) tree(k, page(cycle[0]));
      const int last = page(cycle[L - 1]);
      emit(cycle[0], last, page(cycle[0]));
      for (int k = 1; k < L; ++k) {
        const int over = page(cycle[k - 1]);  // the cycle's own move last: until then `over` may hold what is kept
        emit(cycle[k], over, over);
        push(PageMove{page(cycle[k]), over}, over);
      }
      push(PageMove{-1, last}, last);
    }
  }

 private:
  std::vector<PageMove> given;             // by source
  std::vector<int32_t> first;              // [hubs + 1] into `given`
  std::vector<int32_t> parent;
  std::vector<std::vector<int32_t>> kids;  // hubs whose page becomes this hub's page
  std::vector<int32_t> order;
  std::vector<char> seen;
  int32_t keep = -1;   // of the run that moves are being added to
  bool loose = false;  // its moves are independent of each other

  int page(int h) const { return given[first[h]].src; }
  int hub_of(int32_t p) const {
    int lo = 0, hi = (int)first.size() - 1;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (page(mid) < p) lo = mid + 1;
      else hi = mid;
    }
    return lo < (int)first.size() - 1 && page(lo) == p ? lo : -1;
  }
  void begin(int32_t keep_page, bool any_order) {
    keep = keep_page;
    loose = any_order;
    start();
  }
  void start() {  // a run in the current launch, or in a new one
    if (launches.empty() || launches.back().n_moves >= FORK_MOVES - 1)  // (one place is for what a cycle puts down)
      launches.push_back(Launch{(int32_t)moves.size(), 0, (int32_t)runs.size(), 0});
    runs.push_back(PageRun{launches.back().n_moves, 0, keep});
    ++launches.back().n_runs;
  }
  void add(PageMove m) {
    moves.push_back(m);
    ++launches.back().n_moves;
    ++runs.back().n;
  }
  void push(PageMove m, int32_t spare) {
    if (launches.back().n_moves >= FORK_MOVES - 1) {
      if (keep >= 0 && spare != keep) {
        add(PageMove{-1, spare});
        keep = spare;
      }
      start();
    } else if (loose && runs.back().n >= FORK_FAN) {
      start();
    }
    add(m);
  }
  void emit(int h, int but_not_to, int32_t spare) {
    for (int i = first[h]; i < first[h + 1]; ++i)
      if (given[i].dst != but_not_to) push(given[i], spare);
  }
  void tree(int root, int32_t spare) {
    order.assign(1, root);
    seen[root] = 1;
    for (size_t i = 0; i < order.size(); ++i)
      for (int k : kids[order[i]]) { seen[k] = 1; order.push_back(k); }
    for (size_t i = order.size(); i-- > 0;) emit(order[i], -1, spare);  // (children stand behind their parents)
  }
};
