// Index code of the paged cache, for the device and (in a test) for the host: which rows of a sequence a call looks at, in
// blocks of 32, how blocks become units of work, and where a row stands.  Whatever the caller's arrays hold, nothing here
// names a place outside them.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define PAGED_HD __host__ __device__ __forceinline__
#else
#define PAGED_HD inline
#endif

namespace beagle {

constexpr int PAGED_BLOCK = 32;            // rows that the attention counts its work in

PAGED_HD int paged_min(int a, int b) { return a < b ? a : b; }
PAGED_HD int paged_max(int a, int b) { return a > b ? a : b; }

// slot `s` of n_slots, -1 if it is none; the length that it may be taken to have; pages of that many rows
PAGED_HD int paged_slot_of(int s, int n_slots) { return (unsigned)s < (unsigned)n_slots ? s : -1; }
PAGED_HD int paged_clamped(int len, int slot_pages, int shift) { return paged_min(paged_max(len, 0), slot_pages << shift); }
PAGED_HD int paged_pages(int rows, int shift) { return (rows + (1 << shift) - 1) >> shift; }

// The rows that the queries of an entry may see: true ones below nt (with a window, the first `sinks` and the last `window` of them),
// drafted ones from nt to n.  In blocks: all of them but `skip` behind the first `lead`, which the window hides whole.
struct PagedRows { int n, nt, window, sinks, lead, skip, blocks; };
PAGED_HD PagedRows paged_rows(int n, int nt, int window, int sinks) {
  PagedRows r;
  r.n = n; r.nt = paged_min(paged_max(nt, 0), n); r.window = window; r.sinks = sinks; r.lead = r.skip = 0;
  if (window > 0) {
    r.lead = (paged_min(sinks, r.nt) + PAGED_BLOCK - 1) / PAGED_BLOCK;
    r.skip = paged_max(paged_max(r.nt - window, 0) / PAGED_BLOCK - r.lead, 0);
  }
  r.blocks = (n + PAGED_BLOCK - 1) / PAGED_BLOCK - r.skip;
  return r;
}
PAGED_HD int paged_block(const PagedRows& r, int i) { return i < r.lead ? i : i + r.skip; }
// some query may see the row (a drafted one: as the tree says)
PAGED_HD bool paged_seen(const PagedRows& r, int row) {
  return row < r.n && (row >= r.nt || r.window == 0 || row < r.sinks || row >= r.nt - r.window);
}
// every row of [first, first + count) is a true one that every query sees
PAGED_HD bool paged_all_seen(const PagedRows& r, int first, int count) {
  return first + count <= r.nt && (r.window == 0 || first + count <= r.sinks || first >= r.nt - r.window);
}

// Units: runs of `chunk` blocks of one entry, at least one per entry.  With chunk at least all / target there are at most
// target + entries of them, and at most 2 * target belong to entries that have several.
PAGED_HD int paged_chunk(int64_t all, int target, int least) {
  int64_t c = (all + target - 1) / target;
  if (c < least) c = least;
  return c < (1 << 24) ? (int)c : 1 << 24;              // (no entry has more blocks: 2^28 rows)
}
PAGED_HD int paged_units(int blocks, int chunk) { return paged_max((blocks + chunk - 1) / chunk, 1); }

// page of a row that paged_seen accepts (any other: -1); -1 where the table names no page of the pool
PAGED_HD int paged_page(const int32_t* table, int row, bool seen, int shift, int n_pages) {
  const int p = seen ? table[row >> shift] : -1;
  return (unsigned)p < (unsigned)n_pages ? p : -1;
}

}  // namespace beagle
