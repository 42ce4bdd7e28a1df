// Index code of the paged cache, for the device and (in a test) for the host: which rows of a sequence a call looks at, in
// blocks of 32, how they are divided among workers, and where a row stands.  Whatever the caller's arrays hold, nothing here
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
  r.blocks = paged_max((n + PAGED_BLOCK - 1) / PAGED_BLOCK - r.skip, 1);     // (an empty entry has one, of rows that nobody sees)
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

// Workers: the blocks of all entries in a row (`all` of them, every entry at least one), cut into equal runs, one for each; an entry of up to
// four blocks is not cut but goes whole to the worker that has its first block.  A worker so has at most two entries in part, its first
// and its last.  Where each entry can be cut for itself into runs of four blocks (or of eight, if an equal share is three blocks at least), with
// a worker for each run, entries count as multiples of the run's length instead: then no worker has two, one behind the other.
// Equal runs / runs of eight, us (8 kv heads of 128 bf16, 64 workers): 40 entries of 150 rows 14.2 / 10.8, 20 with 10 queries each 20.9 / 13.4; below the
// limit the runs would be no slower either: 36 entries 13.9 / 10.7.
constexpr int PAGED_RUN = 2, PAGED_LONG_RUN = 3;         // runs of 1 << PAGED_RUN or 1 << PAGED_LONG_RUN blocks
struct PagedSplit { int64_t all; int workers, shift; bool apart; };
PAGED_HD int paged_runs(int blocks, int shift) { return (blocks + (1 << shift) - 1) >> shift; }
PAGED_HD bool paged_apart(int64_t all, int64_t runs, int shift, int target) {
  return runs <= target && (shift == PAGED_RUN || ((1 << shift) - 5) * (int64_t)target <= all);
}
// `runs`: those of all entries, each for itself; not read unless `apart`
PAGED_HD PagedSplit paged_split(int64_t all, int64_t runs, int shift, bool apart, int target) {
  if (apart) return PagedSplit{runs << shift, (int)runs, shift, true};
  const int64_t n = (all + (1 << PAGED_RUN) - 1) >> PAGED_RUN;
  return PagedSplit{all, n < target ? (int)n : target, PAGED_RUN, false};
}
PAGED_HD int paged_counted(const PagedSplit& s, int blocks) { return s.apart ? paged_runs(blocks, s.shift) << s.shift : blocks; }
// worker w takes blocks paged_cut(w) .. paged_cut(w + 1) - 1 of the row
PAGED_HD int64_t paged_cut(const PagedSplit& s, int w) { return s.apart ? (int64_t)w << s.shift : s.all * w / s.workers; }
PAGED_HD int paged_worker_of(const PagedSplit& s, int64_t block) {
  return (int)(s.apart ? block >> s.shift : ((block + 1) * s.workers - 1) / s.all);
}
// blocks [from, to) of an entry that starts at `start` and has `blocks` fall to the worker of [lo, hi)
struct PagedShare { int from, to; };
PAGED_HD PagedShare paged_share(const PagedSplit& s, int64_t start, int blocks, int64_t lo, int64_t hi) {
  if (blocks <= 1 << s.shift) return start >= lo && start < hi ? PagedShare{0, blocks} : PagedShare{0, 0};
  const int64_t a = start < lo ? lo : start, b = start + blocks < hi ? start + blocks : hi;
  return a < b ? PagedShare{(int)(a - start), (int)(b - start)} : PagedShare{0, 0};
}

// page of a row that paged_seen accepts (any other: -1); -1 where the table names no page of the pool
PAGED_HD int paged_page(const int32_t* table, int row, bool seen, int shift, int n_pages) {
  const int p = table[seen ? row >> shift : 0];          // (no branch: a lane without a row reads the first entry for nothing)
  return seen && (unsigned)p < (unsigned)n_pages ? p : -1;
}

}  // namespace beagle
