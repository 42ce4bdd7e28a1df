// Host build of the index code for picked pages and own rows, under sanitizers.  Reads lines of whole numbers, prints what the code says:
//   pick n nt window sinks n_list shift n_pages list.. | table..   -> lead listed gap, rows, true rows, then the page number at every place
//   from n nt from  -> blocks, then for every row 0 .. n + 40: blocks that hold it * 2 + seen
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
    std::string what, word;
    in >> what;
    std::vector<long long> x;
    std::vector<int32_t> table;
    bool behind = false;
    while (in >> word) {
      if (word == "|") behind = true;
      else if (behind) table.push_back((int32_t)std::stoll(word));
      else x.push_back(std::stoll(word));
    }
    if (what == "pick") {
      const int n = (int)x[0], nt = (int)x[1], shift = (int)x[5];
      std::vector<int32_t> list(x.begin() + 7, x.end());
      const PagedPick p = paged_pick(n, nt, (int)x[2], (int)x[3], (int)x[4], shift);
      const PagedRows r = paged_picked_rows(p, n, nt, shift);
      std::printf("%d %d %d %d %d", p.lead, p.listed, p.gap, r.n, r.nt);
      if (!table.empty())
        for (int i = 0; i < paged_pages(r.n, shift); ++i) {
          if (p.listed > (int)list.size()) return 3;
          // exactly sized copies, so that a read outside them is caught
          std::vector<int32_t> l(list.begin(), list.begin() + p.listed);
          std::printf(" %d", paged_picked_page(p, l.data(), table.data(), i, (int)x[6]));
        }
      std::printf("\n");
    } else {
      const PagedRows r = paged_rows_from((int)x[0], (int)x[1], (int)x[2]);
      std::printf("%d", r.blocks);
      if (x[0] <= 4096) {
        std::vector<int> hold(x[0] + 96, 0);
        for (int i = 0; i < r.blocks; ++i)
          for (int j = 0; j < PAGED_BLOCK; ++j) hold.at(paged_block(r, i) * PAGED_BLOCK + j) += 1;
        for (int row = 0; row < x[0] + 40; ++row) {
          // nothing that is not seen may count as all seen
          if (paged_all_seen(r, row / 32 * 32, 32) && !paged_seen(r, row)) return 4;
          std::printf(" %d", hold.at(row) * 2 + paged_seen(r, row));
        }
      }
      std::printf("\n");
    }
  }
  return 0;
}
