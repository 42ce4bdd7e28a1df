// Host build of the paged cache's index code, under sanitizers.  Reads lines of whole numbers, prints what the code says:
//   rows n nt window sinks   -> number of blocks, then for every row 0 .. n + 40: counted blocks that hold it * 4 + seen * 2 + (its block of 32 is all seen)
//   workers target longest blocks.. -> their number, the run where each entry is cut for itself (else 0), (worker, entry, from, to) of every share, (first, last) worker of every entry
//   page n_pages shift row seen entry.. -> the page
//   slot s n_slots len slot_pages shift -> slot, clamped length, its pages
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>
#include <vector>
#include "../paper_2505_24544_amd/csrc/paged_index.h"
using namespace beagle;

int main() {
  std::string line;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    std::string what;
    in >> what;
    std::vector<long long> x;
    for (long long v; in >> v;) x.push_back(v);
    if (what == "rows") {
      const PagedRows r = paged_rows((int)x[0], (int)x[1], (int)x[2], (int)x[3]);
      std::printf("%d", r.blocks);
      if (x[0] <= 4096) {
        std::vector<int> hold(x[0] + 96, 0);
        for (int i = 0; i < r.blocks; ++i)
          for (int j = 0; j < PAGED_BLOCK; ++j) hold.at(paged_block(r, i) * PAGED_BLOCK + j) += 1;
        for (int row = 0; row < x[0] + 40; ++row)
          std::printf(" %d", hold.at(row) * 4 + paged_seen(r, row) * 2 + paged_all_seen(r, row / 32 * 32, 32));
      }
      std::printf("\n");
    } else if (what == "workers") {
      std::vector<long long> start;
      long long all = 0;
      const int target = (int)x[0], longest = (int)x[1];
      auto runs_of = [&](int shift) {
        long long runs = 0;
        for (size_t i = 2; i < x.size(); ++i) runs += paged_runs((int)x[i], shift);
        return runs;
      };
      for (size_t i = 2; i < x.size(); ++i) all += x[i];
      int shift = PAGED_RUN;
      while (!paged_apart(all, runs_of(shift), shift, target) && shift < longest) ++shift;
      const PagedSplit split = paged_split(all, runs_of(shift), shift, paged_apart(all, runs_of(shift), shift, target), target);
      all = 0;
      for (size_t i = 2; i < x.size(); ++i) {
        start.push_back(all);
        all += paged_counted(split, (int)x[i]);
      }
      std::printf("%d %d", split.workers, split.apart ? 1 << split.shift : 0);
      for (int w = 0; w < split.workers; ++w)
        for (size_t i = 2; i < x.size(); ++i) {
          const PagedShare s = paged_share(split, start[i - 2], (int)x[i], paged_cut(split, w), paged_cut(split, w + 1));
          if (s.from < s.to) std::printf(" %d %d %d %d", w, (int)i - 2, s.from, s.to);
        }
      for (size_t i = 2; i < x.size(); ++i)
        std::printf(" %d %d", paged_worker_of(split, start[i - 2]), paged_worker_of(split, start[i - 2] + x[i] - 1));
      std::printf("\n");
    } else if (what == "page") {
      std::vector<int32_t> table(x.begin() + 4, x.end());
      std::printf("%d\n", paged_page(table.data(), (int)x[2], x[3] != 0, (int)x[1], (int)x[0]));
    } else {
      const int s = paged_slot_of((int)x[0], (int)x[1]), len = paged_clamped((int)x[2], (int)x[3], (int)x[4]);
      std::printf("%d %d %d\n", s, len, paged_pages(len, (int)x[4]));
    }
  }
  return 0;
}
