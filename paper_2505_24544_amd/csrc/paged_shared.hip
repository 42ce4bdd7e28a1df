// Attention of a few queries of each of B sequences whose first rows are the same within groups of them (branches of one
// sequence, users under one prompt): the common rows are fetched once for all queries of the group, every sequence's own rows once for its own.
//
//   over rows P (common) and T (own):  m = max(m_P, m_T),  l = l_P 2^(m_P - m) + l_T 2^(m_T - m),  o = (o_P 2^(m_P - m) + o_T 2^(m_T - m)) / l
//
// Bound: the rows' bytes where groups have few query rows, their products where many (see attend_wide); of little work the three launches and their trips to
// memory, some 14 us.  Measured (MI355X, bf16, a graph's replays): 12 entries of 10 queries under a tree, 40 heads, 3 groups of up to 6000 common rows, up to
// 500 own (340 MB) 95 us, its second launch 78 at 4.4 TB/s; 32 entries of a query, 32 / 8 heads, 4000 common, up to 700 own (69 MB) 31 us, its second launch 20.
// Each entry by itself they would read 1.0 and 0.6 GB.  Of few common rows paged_attend, one launch or two, takes less though it reads them for every entry: 4 entries
// of a query 340 rows 8.3 us and here 15.8, 4000 16.5 / 20.4, 16000 32.1 / 30.5; 16 entries of 1000 17.6 / 18.5, 2000 23.9 / 20.2; 64 of 300 and 200 own 25.4 / 27.1,
// 1000 39.3 / 28.5.
//
// Three launches.  The first, one workgroup, divides the work into units: some blocks of 32 rows for a few tiles of 16 query rows, of a
// group's common rows or of an entry's own.  In the second as many workgroups as fit take units, those that are done take more; each unit
// leaves its sums in the workspace, in a place of its own.  The third joins every query row's sums in the order of the rows.
#include "paged_attend.h"
#include "attn_tiles.h"

namespace beagle {
namespace {

constexpr int PLAN_THREADS = 1024;
// The workgroups of the second launch: of four waves, two on a compute unit, or where groups have many query rows (bf16) of eight.  With `cols`
// query rows in a wide unit, and what a block of 32 rows takes one of them, in tenths of a microsecond: common rows for one block of query rows, own rows.
template <int WAVES> struct Work {
  static constexpr int workgroups = 256 * 8 / WAVES, cols = 16 * WAVES, stages = WAVES / 2;
  static constexpr int common = WAVES == 8 ? 3 : 5, wide = 8, own = WAVES == 8 ? 4 : 6;
};

struct Unit {
  int32_t own, b, slot, rb;                // own rows of entry b, or a group's that begins with entry b; which block of query rows
  int32_t first, last, n, nt;              // blocks; rows in all, true ones
  int32_t from, entries;                   // own rows: from this row on; of how many entries the query rows are
  int64_t part;                            // row of the parts, per kv head
};
// where the parts of an entry's query rows are: rows [common + i * stride + ..], i < n_common, [own + i * R + ..], i < n_own
struct Where { int64_t common, own; int32_t stride, offset, n_common, n_own; };
constexpr int QUEUE = 16;                  // words from one queue's count of units taken to the next
struct Plan { int32_t units, pad[63]; };

struct SharedLayout { size_t queue, units, where, ml, part, total; int64_t max_units, rows; };

struct Shares {
  PagedAttnArgs a;
  const int32_t *group_first, *n_shared;
  int32_t queues, workgroups, waves;       // queues of units; workgroups, and the waves of one, which a unit has blocks for at least
  int32_t cost_common, cost_wide, cost_own;
  float workers;                           // of a kv head
  int32_t groups, common_cols, own_blocks;                   // query rows of a unit of common rows; blocks of query rows of an entry
  int32_t wide;                            // query rows of a wide unit, which groups of more than common_cols have (0: none has)
  Plan* plan; int32_t* queue; Unit* units; Where* where;
};

// Sum of v over the threads before this one, and over all; `tmp` holds one value for each wave
template <class T>
__device__ __forceinline__ T sum_before(T v, T* tmp, T* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T upto = v;
  for (int i = 1; i < 64; i *= 2) { const T o = __shfl_up(upto, i); if (lane >= i) upto += o; }
  __syncthreads();
  if (lane == 63) tmp[wave] = upto;
  __syncthreads();
  T before = upto - v, sum = 0;
  for (int w = 0; w < PLAN_THREADS / 64; ++w) { if (w < wave) before += tmp[w]; sum += tmp[w]; }
  *all = sum;
  return before;
}

__device__ __forceinline__ bool is_wide(const Shares& s, int entries) { return s.wide && (int64_t)entries * s.a.M * (s.a.H / s.a.G) > s.common_cols; }
__device__ __forceinline__ int cols_of(const Shares& s, int entries) {
  const int each = is_wide(s, entries) ? s.wide : s.common_cols;
  return (entries * s.a.M * (s.a.H / s.a.G) + each - 1) / each;
}
__device__ __forceinline__ int cost_of(const Shares& s, int entries) { return is_wide(s, entries) ? s.cost_wide : s.cost_common; }
struct Group { int lo, entries, slot, n, blocks, cols; };
__device__ __forceinline__ Group group_of(const Shares& s, const int* first, int g) {
  Group r = {};
  if (g >= s.groups) return r;
  r.lo = first[g];
  r.entries = first[g + 1] - r.lo;
  if (r.entries <= 0) return r;
  r.slot = paged_slot(s.a.c, s.a.slots, r.lo);
  r.n = min(min(max(s.n_shared[g], 0), paged_len(s.a.c, r.slot)), s.a.bound);
  r.blocks = (r.n + PAGED_BLOCK - 1) / PAGED_BLOCK;
  r.cols = r.blocks ? cols_of(s, r.entries) : 0;
  return r;
}
// What a unit is to take: so much that each worker has one, or of long work two, so that those who are done early have something to take.  (Cutting n items
// into equal lengths makes half a unit more of each; but no unit takes a third more than an equal share: 64 entries of 700 own rows behind 4000 common ones
// 57 us with twice a share, 52 so, 256 in 4 groups 149 / 137.)
constexpr float LONG = 240.f;
__device__ __forceinline__ float aimed(float work, float items, float workers) {
  const float units = work > LONG * workers ? 2.f * workers : workers;
  return work / fmaxf(units - 0.5f * items, 0.75f * workers);
}
// units of up to `aim` that so many blocks are cut into
__device__ __forceinline__ int cuts_of(int blocks, float aim, int cost, int least) {
  const int length = (int)fminf(fmaxf(aim / (float)cost, (float)least), (float)(1 << 28));
  return (int)((unsigned)(blocks + length - 1) / (unsigned)length);
}
// first block of cut i of n; common rows are cut between pairs of blocks, which the wide units take at a time
__device__ __forceinline__ int cut_at(int blocks, int i, int n, bool own) {
  return own ? (int)((int64_t)blocks * i / n) : min((int)((int64_t)((blocks + 1) / 2) * i / n) * 2, blocks);
}

// the group that entry b is in: -1 if it is in none
__device__ __forceinline__ int group_with(const int* first, int groups, int b) {
  if (b < first[0] || b >= first[groups]) return -1;
  int lo = 0, hi = groups;                 // first[lo] <= b < first[hi]
  while (hi - lo > 1) { const int m = (lo + hi) / 2; if (first[m] <= b) lo = m; else hi = m; }
  return lo;
}
struct Own { int slot, n, nt, from, blocks; };
__device__ __forceinline__ Own own_of(const Shares& s, const int* first, int b) {
  Own r = {};
  if (b >= s.a.B) return r;
  r.slot = paged_slot(s.a.c, s.a.slots, b);
  r.n = min(paged_len(s.a.c, r.slot), s.a.bound);
  r.nt = min(max(s.a.n_true ? s.a.n_true[b] : INT32_MAX, 0), r.n);
  const int g = group_with(first, s.groups, b);
  r.from = g < 0 ? 0 : min(max(s.n_shared[g], 0), r.nt);
  r.blocks = r.n > r.from ? paged_rows_from(r.n, r.nt, r.from).blocks : 0;
  return r;
}

__global__ __launch_bounds__(PLAN_THREADS) void paged_shared_plan_kernel(Shares s) {
  __shared__ int first[PAGED_MAX_BATCH + 1];
  __shared__ int64_t tmp[PLAN_THREADS / 64];
  __shared__ int tops[PLAN_THREADS / 64];
  __shared__ int base[PLAN_THREADS + 1];   // units before each of the groups, or entries, at hand
  __shared__ int64_t rows[PLAN_THREADS];
  __shared__ union { Group group[PLAN_THREADS]; Own own[PLAN_THREADS]; } held;       // those at hand
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t R = (int64_t)s.a.M * (s.a.H / s.a.G);
  // the groups' first entries, each at least the one before
  int most = 0;
  for (int g0 = 0; g0 <= s.groups; g0 += PLAN_THREADS) {
    int v = g0 + tid <= s.groups ? min(max(s.group_first[g0 + tid], 0), s.a.B) : 0;
    for (int i = 1; i < 64; i *= 2) { const int o = __shfl_up(v, i); if (lane >= i) v = max(v, o); }
    if (lane == 63) tops[wave] = v;
    __syncthreads();
    v = max(v, most);
    for (int w = 0; w < PLAN_THREADS / 64; ++w) { if (w < wave) v = max(v, tops[w]); most = max(most, tops[w]); }
    if (g0 + tid <= s.groups) first[g0 + tid] = v;
    __syncthreads();
  }
  // what there is to do, and from it what a unit is to take
  int64_t mine = 0, items = 0, work, sum;
  const Group group0 = group_of(s, first, tid);              // (in most calls all that there are)
  const Own own0 = own_of(s, first, tid);
  for (int g = tid; g < s.groups; g += PLAN_THREADS) {
    const Group x = g == tid ? group0 : group_of(s, first, g);
    mine += (int64_t)x.blocks * x.cols * cost_of(s, x.entries);
    items += x.cols;
  }
  for (int b = tid; b < s.a.B; b += PLAN_THREADS) {
    const int n = b == tid ? own0.blocks : own_of(s, first, b).blocks;
    mine += (int64_t)n * s.own_blocks * s.cost_own;
    items += n ? s.own_blocks : 0;
  }
  sum_before(mine, tmp, &work);
  sum_before(items, tmp, &sum);
  const float aim = aimed((float)work, (float)sum, s.workers);
  if (tid < s.queues) s.queue[tid * QUEUE] = s.workgroups / s.queues;

  int units = 0;
  int64_t parts = 0;
  for (int g0 = 0; g0 < s.groups; g0 += PLAN_THREADS) {
    const Group x = g0 == 0 ? group0 : group_of(s, first, g0 + tid);
    held.group[tid] = x;
    const int cuts = cuts_of(x.blocks, aim, cost_of(s, x.entries), s.waves);
    int64_t all;
    const int64_t at = sum_before((int64_t)cuts * x.cols, tmp, &all), row = sum_before(cuts * x.entries * R, tmp, &sum);
    base[tid] = (int)at; rows[tid] = parts + row;
    if (tid == 0) base[PLAN_THREADS] = (int)all;
    __syncthreads();
    // units of each group: cut after cut of its rows, those of a cut one behind the other
    for (int u = tid; u < (int)all; u += PLAN_THREADS) {
      const int i = group_with(base, PLAN_THREADS, u);
      const Group y = held.group[i];
      const int n = cuts_of(y.blocks, aim, cost_of(s, y.entries), s.waves), cut = (u - base[i]) / y.cols;
      s.units[units + u] = Unit{0, y.lo, y.slot, (u - base[i]) % y.cols, cut_at(y.blocks, cut, n, false), cut_at(y.blocks, cut + 1, n, false),
                                y.n, y.n, 0, y.entries, rows[i] + cut * y.entries * R};
    }
    const int last = min(g0 + PLAN_THREADS, s.groups);
    for (int b = first[g0] + tid; b < first[last]; b += PLAN_THREADS) {
      const int g = group_with(first, s.groups, b);
      const Group y = held.group[g - g0];
      Where* w = s.where + b;
      w->common = rows[g - g0]; w->stride = (int)(y.entries * R); w->offset = (int)((b - y.lo) * R);
      w->n_common = cuts_of(y.blocks, aim, cost_of(s, y.entries), s.waves);
    }
    units += (int)all; parts += sum;
    __syncthreads();
  }
  for (int b0 = 0; b0 < s.a.B; b0 += PLAN_THREADS) {
    const int b = b0 + tid;
    const Own x = b0 == 0 ? own0 : own_of(s, first, b);
    held.own[tid] = x;
    const int cuts = cuts_of(x.blocks, aim, s.cost_own, s.waves);
    int64_t all;
    const int64_t at = sum_before((int64_t)cuts * s.own_blocks, tmp, &all), row = sum_before(cuts * R, tmp, &sum);
    base[tid] = (int)at; rows[tid] = parts + row;
    if (tid == 0) base[PLAN_THREADS] = (int)all;
    __syncthreads();
    for (int u = tid; u < (int)all; u += PLAN_THREADS) {
      const int i = group_with(base, PLAN_THREADS, u);
      const Own y = held.own[i];
      const int n = cuts_of(y.blocks, aim, s.cost_own, s.waves), cut = (u - base[i]) / s.own_blocks;
      s.units[units + u] = Unit{1, b0 + i, y.slot, (u - base[i]) % s.own_blocks, cut_at(y.blocks, cut, n, true), cut_at(y.blocks, cut + 1, n, true),
                                y.n, y.nt, y.from, 1, rows[i] + cut * R};
    }
    if (b < s.a.B) {
      Where* w = s.where + b;
      w->own = rows[tid]; w->n_own = cuts;
      if (group_with(first, s.groups, b) < 0) { w->common = 0; w->stride = w->offset = w->n_common = 0; }
    }
    units += (int)all; parts += sum;
    __syncthreads();
  }
  if (tid == 0) s.plan->units = units;
}

// The same by one wave, where everything is counted in 32 bits: lane b has entry b, lane g group g.
constexpr int WAVE_ENTRIES = 64, WAVE_ROWS = 1 << 15, WAVE_BOUND = 1 << 20;      // entries (and groups: one less), query rows of all, rows of a sequence
// the last of the 64 numbers, in ascending order, that is not above v
__device__ __forceinline__ int last_upto(const int* at, int v) {
  int i = 0;
#pragma unroll
  for (int k = 32; k > 0; k /= 2)
    if (at[i + k] <= v) i += k;
  return i;
}
__global__ __launch_bounds__(64) void paged_shared_small_plan_kernel(Shares s) {
  // of each lane's group and entry: units before, blocks, cuts, .. (of those without a unit, what comes next has the same number before it)
  enum { GROUP_AT, GROUP_LO, GROUP_ENTRIES, GROUP_SLOT, GROUP_N, GROUP_BLOCKS, GROUP_COLS, GROUP_CUTS, GROUP_ROW,
         OWN_AT, OWN_SLOT, OWN_N, OWN_NT, OWN_FROM, OWN_BLOCKS, OWN_CUTS, OWN_ROW, FIELDS };
  __shared__ int f[FIELDS][64];
  const int lane = threadIdx.x, at = min(lane, s.a.B - 1), g_at = min(lane, s.groups - 1), R = s.a.M * (s.a.H / s.a.G);
  auto of = [](int v, int l) { return __builtin_amdgcn_readlane(v, l); };
  const int first = s.group_first[g_at], next = s.group_first[g_at + 1], shared = max(s.n_shared[g_at], 0);
  const int n_true = s.a.n_true ? s.a.n_true[at] : INT32_MAX, slot = paged_slot(s.a.c, s.a.slots, at);
  if (lane < s.queues) s.queue[lane * QUEUE] = s.workgroups / s.queues;
  const int len = s.a.c.lens[max(slot, 0)];
  const int n = lane < s.a.B && slot >= 0 ? min(paged_clamped(len, s.a.c.W, s.a.c.shift), s.a.bound) : 0, nt = min(max(n_true, 0), n);
  const int lo = max_upto(lane < s.groups ? min(max(first, 0), s.a.B) : 0), hi = lane < s.groups ? max(lo, min(max(next, 0), s.a.B)) : lo;
  int common = 0, in_group = -1;           // rows that this lane's entry has in common with others; its group
#pragma unroll 1
  for (int g = 0; g < s.groups; ++g)
    if (lane >= of(lo, g) && lane < of(hi, g)) { common = of(shared, g); in_group = g; }
  const int from = min(common, nt), own_blocks = n > from ? paged_rows_from(n, nt, from).blocks : 0;
  const int lead = min(lo, s.a.B - 1), entries = hi - lo, group_n = min(shared, __shfl(n, lead)), group_slot = __shfl(slot, lead);
  const int blocks = entries > 0 ? (group_n + PAGED_BLOCK - 1) / PAGED_BLOCK : 0, cols = blocks ? cols_of(s, entries) : 0, cost = cost_of(s, entries);
  const int work = sum_upto(blocks * cols * cost + own_blocks * s.own_blocks * s.cost_own), items = sum_upto(cols + (own_blocks ? s.own_blocks : 0));
  const float all = (float)of(work, 63), least = all / s.workers;
  float aim = aimed(all, (float)of(items, 63), s.workers);
  if (all <= LONG * s.workers) {
    // One round of units: the least aim, to 3 %, that makes no more units than workers, if 2.5 times an equal share does.  (32 entries, 4000 common rows, 700
    // own: 37 us by the formula, 31 so; 2000 and 400: 29 / 26.  A unit of the formula's more than workers is a second round.)
    auto fits = [&](float aim) {             // (divided roughly)
      auto cuts = [&](int blocks, int cost) {
        const float length = floorf(fmaxf(aim * __builtin_amdgcn_rcpf((float)cost), (float)s.waves));
        return (int)ceilf((float)blocks * __builtin_amdgcn_rcpf(length) * (1.f - 0x1p-18f));
      };
      return (float)of(sum_upto(cuts(blocks, cost) * cols + cuts(own_blocks, s.cost_own) * (own_blocks ? s.own_blocks : 0)), 63) <= s.workers;
    };
    if (fits(2.5f * least)) {
      aim = 2.5f * least;
      float below = least;                   // (does not fit, or is as good)
      if (fits(least)) aim = least;
#pragma unroll 1
      for (int i = 0; i < 5 && aim > 1.03f * below; ++i) {
        const float mid = __builtin_amdgcn_sqrtf(below * aim);
        if (fits(mid)) aim = mid;
        else below = mid;
      }
    }
  }
  const int cuts = cuts_of(blocks, aim, cost, s.waves), own_cuts = cuts_of(own_blocks, aim, s.cost_own, s.waves);
  const int uc = cuts * cols, uo = own_cuts * s.own_blocks, rc = cuts * entries * R, ro = own_cuts * R;
  const int uc_upto = sum_upto(uc), uo_upto = sum_upto(uo), rc_upto = sum_upto(rc), common_units = of(uc_upto, 63), units = common_units + of(uo_upto, 63);
  const int row = rc_upto - rc, own_row = of(rc_upto, 63) + sum_upto(ro) - ro;
  f[GROUP_AT][lane] = uc_upto - uc; f[GROUP_LO][lane] = lo; f[GROUP_ENTRIES][lane] = entries; f[GROUP_SLOT][lane] = group_slot; f[GROUP_N][lane] = group_n;
  f[GROUP_BLOCKS][lane] = blocks; f[GROUP_COLS][lane] = cols; f[GROUP_CUTS][lane] = cuts; f[GROUP_ROW][lane] = row;
  f[OWN_AT][lane] = common_units + uo_upto - uo; f[OWN_SLOT][lane] = slot; f[OWN_N][lane] = n; f[OWN_NT][lane] = nt; f[OWN_FROM][lane] = from;
  f[OWN_BLOCKS][lane] = own_blocks; f[OWN_CUTS][lane] = own_cuts; f[OWN_ROW][lane] = own_row;
  __syncthreads();
  if (lane == 0) s.plan->units = units;
  if (lane < s.a.B) {
    const int g = max(in_group, 0);
    s.where[lane] = Where{f[GROUP_ROW][g], own_row, f[GROUP_ENTRIES][g] * R, (lane - f[GROUP_LO][g]) * R, in_group < 0 ? 0 : f[GROUP_CUTS][g], own_cuts};
  }
#pragma unroll 1
  for (int u = lane; u < units; u += 64) {
    const bool own = u >= common_units;
    const int i = last_upto(f[own ? OWN_AT : GROUP_AT], u), each = own ? s.own_blocks : f[GROUP_COLS][i];
    const int k = u - f[own ? OWN_AT : GROUP_AT][i], cut = (int)((unsigned)k / (unsigned)each), of_all = f[own ? OWN_CUTS : GROUP_CUTS][i];
    const int all = f[own ? OWN_BLOCKS : GROUP_BLOCKS][i], es = own ? 1 : f[GROUP_ENTRIES][i];
    s.units[u] = Unit{own, own ? i : f[GROUP_LO][i], f[own ? OWN_SLOT : GROUP_SLOT][i], k - cut * each, cut_at(all, cut, of_all, own),
                      cut_at(all, cut + 1, of_all, own), f[own ? OWN_N : GROUP_N][i], f[own ? OWN_NT : GROUP_N][i], own ? f[OWN_FROM][i] : 0, es,
                      (int64_t)f[own ? OWN_ROW : GROUP_ROW][i] + (int64_t)cut * es * R};
  }
}

// Common rows for 64 or 128 query rows of a group that has more of them (bf16): tiles of 64 rows go through a ring of LDS stages; half of the waves
// take 32 query rows each against a tile's first half, half of them against its second.  As the training forward, but for the scale in two parts,
// rows that come from pages, and probabilities in three terms that add up to them exactly (see attend_entry).  Infinite values, rows with what is no
// number that some queries do not see, values that leave a float's range times a probability above one, and pages that are none, are not looked for: where
// they show in the result, which is not finite then (or a page's number was none), `false` comes back, and the caller has the unit done row by row.
//
// Bound by the matrix pipe: four products of d for a row and query, 134 G (multiplications and additions) for 64 entries of 4 queries of 32 heads over 16000
// common rows of 8 kv heads.  These take 149 us with the other two launches' 13: 0.98 of the 1.20 PFLOP/s that a product of 8192^3 reaches.
// (Four waves, 64 query rows, two stages: 179 us.)
constexpr int TILE_ROWS = 64;
constexpr int NUMBERS = 2048;              // page numbers that are held at a time
template <int WAVES> struct WideShared { bf16_t stage[Work<WAVES>::stages][2][TILE_ROWS * tiles::HD]; int pages[NUMBERS]; };
template <int WAVES>
__device__ __forceinline__ bool attend_wide(const PagedAttnArgs& a, WideShared<WAVES>& sh, const Item& item, int b, int slot, int n, int first, int last,
                                            int head, int cb) {
  using namespace tiles;
  constexpr int STAGES = Work<WAVES>::stages, COLS = Work<WAVES>::cols, HALF = WAVES / 2, CHUNKS = 16 / WAVES;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));            // what is made of it belongs to this unit: kept for the next one it would take registers
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5, ql = lane & 31;
  const int qw = wave % HALF, kw = wave / HALF * 32;                // this wave's query rows, and its first row of a tile
  const int rep = a.H / a.G, R = item.R, r = cb * COLS + qw * 32 + ql;
  const uint32_t row_bytes = (uint32_t)a.G * HD * 2, page_bytes = row_bytes << a.c.shift;          // (the launcher sees to 32 bits)
  const addr_t zero = (addr_t)zero_row;
  const int32_t* table = a.c.table + (int64_t)max(slot, 0) * a.c.W;
  const int shift = a.c.shift, in_page = (1 << shift) - 1;
  const int row0 = first * PAGED_BLOCK, rows_end = min(last * PAGED_BLOCK, n), tiles_ = (rows_end - row0 + TILE_ROWS - 1) / TILE_ROWS;
  // tiles whose page numbers are held: they begin with one of the numbers' first row at most a page before it
  const int held = max(((NUMBERS - 1) << min(shift, 16)) / TILE_ROWS, 1);
  bool bad = false;
  int page0 = 0;
  auto look = [&](int t0, int t1) {
    page0 = (row0 + t0 * TILE_ROWS) >> shift;
    const int end = t1 < tiles_ ? (row0 + t1 * TILE_ROWS - 1) >> shift : (rows_end - 1) >> shift;
    for (int i = page0 + tid; i <= end; i += 64 * WAVES) {
      const int number = table[i];
      const bool none = (unsigned)number >= (unsigned)a.c.P;
      bad |= none;
      sh.pages[i - page0] = none ? 0 : number;
    }
  };
  const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uintptr_t)(lds_void_ptr)sh.stage[0][0]);
  // this thread fetches its chunk of rows tid / 16 + 4 WAVES i of a tile (swz is the same for all of them; rows behind the end are the last one again)
  const addr_t kbase = (addr_t)a.c.k + (int64_t)head * HD * 2 + ((tid & 15) ^ swz(tid >> 4)) * 16, to_v = (addr_t)a.c.v - (addr_t)a.c.k;
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int row = min(row0 + t * TILE_ROWS + (tid >> 4) + 4 * WAVES * i, rows_end - 1), number = sh.pages[(row >> shift) - page0];
      const addr_t k = kbase + (uint64_t)(uint32_t)number * page_bytes + (uint32_t)(row & in_page) * row_bytes, v = k + to_v;
      const uint32_t dst = lds0 + (uint32_t)((t % STAGES * 2 * TILE_ROWS * HD + (i * WAVES + wave) * 512) * 2);
      load_to_lds(k, dst);
      load_to_lds(v, dst + TILE_ROWS * HD * 2);
    }
  };
  bf16x8_t qf[HD / 16];
  {
    const addr_t p = (addr_t)a.q + (((int64_t)b * a.M + r / rep) * a.H + head * rep + r % rep) * HD * 2;
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) qf[s] = __builtin_bit_cast(bf16x8_t, load16(r < R ? p + 32 * s + 16 * hf : zero));
  }
  const int at = b + min(r / (a.M * rep), item.entries - 1), nt = a.n_true ? a.n_true[at] : INT32_MAX;
  const int limit = min(min(max(nt, 0), rows_end), min(paged_len(a.c, paged_slot(a.c, a.slots, at)), a.bound));
  // the least of the limits of this wave's query rows that see anything; the others are cleared at the end
  int least = limit > 0 ? limit : INT32_MAX;
#pragma unroll
  for (int i = 1; i < 32; i *= 2) least = min(least, __shfl_xor(least, i));
  least = __builtin_amdgcn_readfirstlane(least);
  f32x16_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  const FragOffs fo = make_frag_offs(lane);
  auto scaled = [&](float x, float less) { return fmaf(x, a.c2_low, fmaf(x, a.c2, -less)); };
  auto step = [&](int t) BEAGLE_INLINE_LAMBDA {
    const bf16_t *ks = sh.stage[t % STAGES][0] + kw * HD, *vs = ks + TILE_ROWS * HD;
    f32x16_t st;
#pragma unroll
    for (int e = 0; e < 16; ++e) st[e] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
    bf16x8_t kf[HD / 16];
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) kf[s] = row_frag(ks, fo, 0, s);
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s], st, 0, 0, 0);
    pipeline_reads_mfma<HD / 16, 1>();
    __builtin_amdgcn_sched_barrier(0);
    const int j0 = row0 + t * TILE_ROWS + kw;                  // register e is row j0 + 8 (e / 4) + 4 hf + e % 4
    if (j0 + 32 > least) {
      const int rel = limit - j0 - 4 * hf;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (8 * (e >> 2) + (e & 3) >= rel) st[e] = -INFINITY;
    }
    float mx = st[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, st[e]);
    mx = scaled(half_pair_max(mx), 0.f);
    // (the reference moves where the maximum has grown by more than 2^8: float sums and terms have room for that)
    const bool grow = mx - m > 8.f;
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
      const float now = grow ? mx : m, alpha = grow ? exp2_fast(m - now) : 1.f;
      l *= alpha;
      m = now;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
    }
    const float safe = m == -INFINITY ? 0.f : m;
    union Term { uint32_t u[4]; bf16x8_t v; } term[3][2];
    auto terms = [&](int h) BEAGLE_INLINE_LAMBDA {
#pragma unroll
      for (int e = 8 * h; e < 8 * h + 8; e += 2) {
        const float p0 = exp2_fast(scaled(st[e], safe)), p1 = exp2_fast(scaled(st[e + 1], safe));
        l += p0 + p1;
        uint32_t x = __float_as_uint(p0), y = __float_as_uint(p1);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          term[k][h].u[(e & 7) >> 1] = __builtin_amdgcn_perm(y, x, 0x07060302u);
          if (k == 2) break;
          x = __float_as_uint(__uint_as_float(x) - __uint_as_float(x & 0xffff0000u));
          y = __float_as_uint(__uint_as_float(y) - __uint_as_float(y & 0xffff0000u));
        }
      }
    };
    auto values = [&](int h, const bf16x8_t (&w)[4]) BEAGLE_INLINE_LAMBDA {
#pragma unroll
      for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[c], term[k][h].v, o[c], 0, 0, 0);
    };
    bf16x8_t w0[4], w1[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) w0[c] = tr_frag(vs, fo, 0, c);
    terms(0);
    __builtin_amdgcn_sched_barrier(0);
    // the first sixteen rows' products run behind the second's probabilities
#pragma unroll
    for (int c = 0; c < 4; ++c) w1[c] = tr_frag(vs, fo, 16, c);
    values(0, w0);
    terms(1);
#pragma unroll
    for (int i = 0; i < 12; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i < 8) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, 7, 0);       // vector, transcendental
    }
    __builtin_amdgcn_sched_barrier(0);
    values(1, w1);
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll 1
  for (int t0 = 0; t0 < tiles_; t0 += held) {
    const int t1 = min(t0 + held, tiles_);
    look(t0, t1);
    __syncthreads();
#pragma unroll 1
    for (int t = t0; t < min(t0 + STAGES - 1, t1); ++t) fetch(t);
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
      // tile t is there when all but the requests of the tiles behind it are back (2 CHUNKS for each), in all waves; then nobody reads tile t - 1
      // any more, whose place the next one takes
      if (STAGES > 3 && t + 2 < t1) wait_vmem_n<4 * CHUNKS>();
      else if (STAGES > 2 && t + 1 < t1) wait_vmem_n<2 * CHUNKS>();
      else wait_vmem_n<0>();
      lds_barrier();
      if (t + STAGES - 1 < t1) fetch(t + STAGES - 1);
      step(t);
    }
    __syncthreads();
  }

  l = half_pair_sum(l);
  if (limit <= 0) {
    m = -INFINITY; l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  }
  // the second half's result joins the first's
  float4* po = (float4*)sh.stage[0][0] + qw * 64 + lane;       // [16][HALF][64 lanes]: half of the stages
  float2* pml = (float2*)sh.stage[STAGES / 2][0] + qw * 64 + lane;
  int* flag = sh.pages;
  if (tid == 0) *flag = 0;
  __syncthreads();
  if (kw) {
#pragma unroll
    for (int i = 0; i < 16; ++i) po[64 * HALF * i] = float4{o[i >> 2][4 * (i & 3)], o[i >> 2][4 * (i & 3) + 1], o[i >> 2][4 * (i & 3) + 2], o[i >> 2][4 * (i & 3) + 3]};
    *pml = float2{m, l};
    if (bad) *flag = 1;
  }
  __syncthreads();
  if (!kw) {
    const float2 ml = *pml;
    const float now = fmaxf(m, ml.x), safe = now == -INFINITY ? 0.f : now;
    const float w0 = exp2_fast(m - safe), w1 = exp2_fast(ml.x - safe);
    m = now;
    l = l * w0 + ml.y * w1;
    float sum = l;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float4 v = po[64 * HALF * i];
      const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) { o[i >> 2][4 * (i & 3) + e] = o[i >> 2][4 * (i & 3) + e] * w0 + w[e] * w1; sum += o[i >> 2][4 * (i & 3) + e]; }
    }
    if (bad || (r < R && !(fabsf(sum) < INFINITY))) *flag = 1;
  }
  __syncthreads();
  const bool whole = *flag == 0;
  if (whole && !kw && r < R) {
    float* row = a.part + (item.part_row + r) * HD;
#pragma unroll
    for (int i = 0; i < 16; ++i)                               // channels 32 (i / 4) + 8 (i % 4) + 4 hf ..
      *(f32x4*)(row + 32 * (i >> 2) + 8 * (i & 3) + 4 * hf) =
          f32x4{o[i >> 2][4 * (i & 3)], o[i >> 2][4 * (i & 3) + 1], o[i >> 2][4 * (i & 3) + 2], o[i >> 2][4 * (i & 3) + 3]};
    if (hf == 0) *(float2*)(a.ml + (item.part_row + r) * 2) = make_float2(m, l);
  }
  return whole;
}

// The workgroups that have the same number modulo eight share a die and its cache: those of one head, as far as heads go.
template <bool BF16, int NH, int RTC, int RTO, bool TREE, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 8 / WAVES) void paged_shared_kernel(Shares s) {
  using S = Shape<BF16, NH>;
  __shared__ __attribute__((aligned(1024))) union {
    WideShared<WAVES> wide[BF16 ? 1 : 0];
    Shared<S, RTC, WAVES, PREFIX> common;
    Shared<S, RTO, WAVES, SUFFIX> own;
  } shared;
  auto wave = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  // one queue for each die that has heads of its own: of every unit, its heads
  const int queue = blockIdx.x % s.queues, heads = s.a.G / s.queues, units = wave(s.plan->units);
#pragma unroll 1
  for (int64_t i = blockIdx.x / s.queues; i < (int64_t)units * heads;) {
    const int u = (int)((uint32_t)i / (uint32_t)heads), head = (int)((uint32_t)i % (uint32_t)heads) * s.queues + queue;
    const Unit x = s.units[u];
    // what comes next is asked for now, and known when this unit is done
    int next = 0;
    if (threadIdx.x == 0) next = __hip_atomic_fetch_add(s.queue + queue * QUEUE, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int R = s.a.M * (s.a.H / s.a.G) * wave(x.entries);
    Item item = {};
    item.R = R; item.entries = wave(x.entries);
    const int64_t part = (int64_t)wave((int)(x.part >> 32)) << 32 | (uint32_t)wave((int)x.part);
    item.part_row = part * s.a.G + (int64_t)head * R;
    const int b = wave(x.b), slot = wave(x.slot), rb = wave(x.rb), first = wave(x.first), last = wave(x.last), n = wave(x.n);
    if (wave(x.own)) {
      attend_entry<BF16, NH, RTO, TREE, WAVES, SUFFIX>(s.a, shared.own, item, b, slot, paged_rows_from(n, wave(x.nt), wave(x.from)), first, last, false, 0,
                                                       head, rb);
    } else {
      int block = rb, blocks = 1;
      if constexpr (BF16)
        if (is_wide(s, item.entries)) {
          const bool done = attend_wide<WAVES>(s.a, shared.wide[0], item, b, slot, n, first, last, head, rb);
          blocks = done ? 0 : WAVES / RTC;
          block = rb * (WAVES / RTC);
        }
#pragma unroll 1
      for (int k = 0; k < blocks; ++k) {
        __syncthreads();
        attend_entry<BF16, NH, RTC, false, WAVES, PREFIX>(s.a, shared.common, item, b, slot, paged_rows(n, n, 0, 0), first, last, false, 0, head, block + k);
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) *(int*)&shared = next;
    __syncthreads();
    i = (uint32_t)wave(*(const int*)&shared);
    __syncthreads();
  }
}

// A query row's parts, in order: those of the common rows, then those of its own.  As in paged_join_kernel.
template <bool BF16, int HDP, int ROWS>
__global__ __launch_bounds__(256) void paged_shared_join_kernel(Shares s) {
  constexpr int LANES = HDP / 4, GROUPS = 256 / LANES, SPLIT = GROUPS / ROWS;
  __shared__ float so[GROUPS][HDP];
  __shared__ float sm[GROUPS], sl[GROUPS];
  const PagedAttnArgs& a = s.a;
  const int rep = a.H / a.G, R = a.M * rep, b = blockIdx.y;
  const Where w = s.where[b];
  const int group = threadIdx.x / LANES, ch = 4 * (threadIdx.x % LANES);
  const int n = blockIdx.x * ROWS + group / SPLIT;         // row of the entry: kv head, then query and head of the group
  const int head = n / R, r = n % R, qi = r / rep, h = head * rep + r % rep;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  auto join = [&](float m2, float l2, f32x4 o2) BEAGLE_INLINE_LAMBDA {
    const float now = fmaxf(m, m2), safe = now == -INFINITY ? 0.f : now;
    const float w0 = exp2_fast(m - safe), w1 = exp2_fast(m2 - safe);
    o = o * w0 + o2 * w1;
    l = l * w0 + l2 * w1;
    m = now;
  };
  const int shares = w.n_common + w.n_own;
  if (n < a.G * R) {
    const int64_t common = w.common * a.G + (int64_t)head * w.stride + w.offset + r, own = w.own * a.G + (int64_t)head * R + r;
    constexpr int AT_ONCE = 4;
    for (int i = group % SPLIT; i < shares; i += SPLIT * AT_ONCE) {
      float2 ml[AT_ONCE];
      f32x4 po[AT_ONCE];
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e) {
        const int k = min(i + e * SPLIT, shares - 1);
        const int64_t row = k < w.n_common ? common + (int64_t)k * w.stride * a.G : own + (int64_t)(k - w.n_common) * R * a.G;
        ml[e] = *(const float2*)(a.ml + row * 2);
        po[e] = *(const f32x4*)(a.part + row * HDP + ch);
      }
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e)
        if (i + e * SPLIT < shares) join(ml[e].x, ml[e].y, po[e]);
    }
  }
  if constexpr (SPLIT > 1) {
    *(f32x4*)&so[group][ch] = o;
    if (ch == 0) { sm[group] = m; sl[group] = l; }
    __syncthreads();
    if (group % SPLIT) return;
#pragma unroll
    for (int i = 1; i < SPLIT; ++i) join(sm[group + i], sl[group + i], *(const f32x4*)&so[group + i][ch]);
  }
  if (n >= a.G * R) return;
  if (ch == 0) a.lse[((int64_t)b * a.H + h) * a.M + qi] = (m + __log2f(l)) * LN2;
  if (ch >= a.d) return;
  o *= l == 0.f ? 0.f : 1.f / l;
  const int64_t at = (((int64_t)b * a.M + qi) * a.H + h) * a.d + ch;
  if constexpr (BF16) *(uint2*)((bf16_t*)a.o + at) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
  else *(f32x4*)((float*)a.o + at) = o;
}

constexpr int COMMON_TILES = 2;            // of 16 query rows in a unit of common rows

// A unit has at least 0.8 of what is aimed at (a length of four blocks or more is rounded down), which is at least half of an equal share: cutting adds at most
// 2.5 units for each worker to those that groups and entries have uncut, and as many query rows to the parts.  (Workgroups of eight waves are half as many,
// with twice the query rows.)
SharedLayout shared_layout(int32_t B, int32_t M, int32_t H, int32_t G) {
  const int64_t R = (int64_t)M * (H / G), cut = (int64_t)Work<4>::workgroups * 5 / 2 / G + 4;
  const Tiles own = tiles_of((int)R);
  SharedLayout l;
  l.max_units = 2 * cut + B + (B * R + 16 * COMMON_TILES - 1) / (16 * COMMON_TILES) + (int64_t)B * own.blocks;
  l.rows = cut * Work<4>::cols + B * R + cut * 16 * own.each + B * R;
  size_t at = sizeof(Plan);
  auto take = [&](size_t n) { const size_t o = at; at = (at + n + 255) / 256 * 256; return o; };
  l.queue = take(8 * QUEUE * sizeof(int32_t));
  l.units = take(l.max_units * sizeof(Unit));
  l.where = take(B * sizeof(Where));
  l.ml = take((size_t)l.rows * G * 2 * sizeof(float));
  l.part = take((size_t)l.rows * G * 128 * sizeof(float));
  l.total = at;
  return l;
}

}  // namespace

size_t paged_shared_ws_bytes(int32_t B, int32_t M, int32_t H, int32_t G) { return shared_layout(B, M, H, G).total; }

void launch_paged_shared(bool bf16, PagedSharedArgs p, void* ws, hipStream_t s) {
  Shares x;
  x.a = p.a;
  set_scale(x.a);
  const SharedLayout l = shared_layout(p.a.B, p.a.M, p.a.H, p.a.G);
  char* at = (char*)ws;
  x.plan = (Plan*)at;
  x.queue = (int32_t*)(at + l.queue);
  x.units = (Unit*)(at + l.units);
  x.where = (Where*)(at + l.where);
  x.a.ml = (float*)(at + l.ml);
  x.a.part = (float*)(at + l.part);
  x.group_first = p.group_first; x.n_shared = p.n_shared; x.groups = p.groups;
  const Tiles own = tiles_of(p.a.M * (p.a.H / p.a.G));
  x.queues = p.a.G % 8 ? 1 : 8;
  const int64_t in_groups = (int64_t)p.a.B * p.a.M * (p.a.H / p.a.G);
  const bool stages = bf16 && ((int64_t)p.a.G * tiles::HD * 2 << p.a.c.shift) < (1ll << 32);
  const bool many = stages && in_groups > (int64_t)Work<8>::cols * p.groups && in_groups * p.a.bound > (int64_t)(3 << 20) * p.groups;
  // Eight waves where a group has on average more query rows than one of their wide units, and those times the rows that a sequence can have pass 3 * 2^20 (8 kv
  // heads, us with 8 / 4 waves): 1024 query rows over 16000 rows 150 / 179, over 4000 65 / 74, 256 over 16000 74 / 78; 512 over 4000 58 / 49, 1024 over
  // 2000 52 / 45, 128 over 4000 44 / 37: there the entries' own rows are as much, whose units are better small and many.  Wide units already from 33
  // query rows on: groups of 40 over 6000 rows, 32 or 40 kv heads: 92 and 81 us, in units of 32 query rows, 113 and 86 (48: as fast).  (The rows are the caller's
  // bound: where it is far above the sequences there are, eight waves come too early, by the figures above up to 9 us.)
  auto work = [&](auto w_) {
    using W = Work<decltype(w_)::value>;
    x.waves = decltype(w_)::value;
    x.workgroups = W::workgroups;
    x.cost_common = W::common; x.cost_wide = W::wide; x.cost_own = W::own;
    x.wide = stages ? W::cols : 0;
  };
  if (many) work(int_c<8>{});
  else work(int_c<4>{});
  x.workers = p.a.G < x.workgroups ? (float)(x.workgroups / p.a.G) : (float)x.workgroups / (float)p.a.G;
  x.common_cols = 16 * COMMON_TILES;
  x.own_blocks = own.blocks;
  const bool by_wave = p.a.B <= WAVE_ENTRIES && p.groups < WAVE_ENTRIES && in_groups <= WAVE_ROWS && p.a.bound <= WAVE_BOUND;
  {
    ProfScope ps("paged_shared_plan", s);
    if (by_wave) hipLaunchKernelGGL(paged_shared_small_plan_kernel, dim3(1), dim3(64), 0, s, x);
    else hipLaunchKernelGGL(paged_shared_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, x);
  }
  const bool narrow = !bf16 && p.a.d <= 64, tree = p.a.n_true != nullptr;
  {
    ProfScope ps("paged_shared", s);
    const dim3 grid((unsigned)x.workgroups), wg((unsigned)(64 * x.waves));
    auto go = [&](auto bf_, auto nh_, auto rt_, auto w_) {
      constexpr bool BF = decltype(bf_)::value != 0;
      constexpr int NH = decltype(nh_)::value, RT = decltype(rt_)::value, W = decltype(w_)::value;
      if (tree) hipLaunchKernelGGL((paged_shared_kernel<BF, NH, COMMON_TILES, RT, true, W>), grid, wg, 0, s, x);
      else hipLaunchKernelGGL((paged_shared_kernel<BF, NH, COMMON_TILES, RT, false, W>), grid, wg, 0, s, x);
    };
    auto with = [&](auto bf_, auto nh_, auto w_) { own.each == 1 ? go(bf_, nh_, int_c<1>{}, w_) : go(bf_, nh_, int_c<2>{}, w_); };
    if (many) with(int_c<1>{}, int_c<1>{}, int_c<8>{});
    else if (bf16) with(int_c<1>{}, int_c<1>{}, int_c<4>{});
    else if (narrow) with(int_c<0>{}, int_c<1>{}, int_c<4>{});
    else with(int_c<0>{}, int_c<2>{}, int_c<4>{});
  }
  ProfScope ps("paged_shared_join", s);
  auto join = [&](auto bf_, auto hdp_) {
    constexpr bool BF = decltype(bf_)::value != 0;
    constexpr int HDP = decltype(hdp_)::value, MANY = 256 / (HDP / 4);
    const int64_t all = (int64_t)p.a.H * p.a.M;
    if (all * p.a.B <= 1024) hipLaunchKernelGGL((paged_shared_join_kernel<BF, HDP, 1>), dim3((unsigned)all, (unsigned)p.a.B), dim3(256), 0, s, x);
    else hipLaunchKernelGGL((paged_shared_join_kernel<BF, HDP, MANY>), dim3((unsigned)((all + MANY - 1) / MANY), (unsigned)p.a.B), dim3(256), 0, s, x);
  };
  if (bf16) join(int_c<1>{}, int_c<128>{});
  else if (narrow) join(int_c<0>{}, int_c<64>{});
  else join(int_c<0>{}, int_c<128>{});
}

}  // namespace beagle
