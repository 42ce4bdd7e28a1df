// What changes a paged cache: appending rows, forking sequences, moving the live pages into another pool.
//
// Everything is whole numbers and copies; a page is free where no slot's table names it (refs[p] == 0), and free pages are taken lowest
// first in the order of the call's entries, so the outcome is a function of the cache's state and the arguments alone.
// Reference counts change by integer atomics, whose order does not show.  Bound: the rows that are copied (HBM), and for
// a few rows the chain of dependent trips to memory in the planning workgroup.
#include "paged.h"

namespace beagle {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
constexpr int PLAN = 1024;                 // threads of a planning workgroup
constexpr int PLAN_WAVES = PLAN / 64;

__device__ __forceinline__ void add_count(int32_t* p, int v) { (void)__hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool is_page(const PagedCache& c, int p) { return (unsigned)p < (unsigned)c.P; }
// a barrier behind which every thread's earlier loads are back, and its stores and atomics have reached the second-level cache (the barrier
// alone waits for none)
__device__ __forceinline__ void all_done() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}
// every thread's earlier stores and atomics are seen by the workgroup's later loads and atomics: they are done, and the vector cache is without what
// it held before (nobody else reads on, so nothing has to be written back for other dies: that fence cost 2 us)
__device__ __forceinline__ void settle() {
  all_done();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
}

// Inclusive sum over the workgroup's threads in order, of K numbers at once; `all` gets the sums of everything.
template <int K> struct Sums { int at[K]; };
template <int K> __device__ __forceinline__ Sums<K> block_scan(Sums<K> v, int (*wave_sums)[PLAN_WAVES], Sums<K>& all) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int k = 0; k < K; ++k) v.at[k] = sum_upto(v.at[k]);
  __syncthreads();                         // (the sums of the call before have been read)
  if (lane == 63)
#pragma unroll
    for (int k = 0; k < K; ++k) wave_sums[k][wave] = v.at[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {            // (a lane for each wave's sum)
    const int x = lane < PLAN_WAVES ? wave_sums[k][lane] : 0, upto = sum_upto(x);
    all.at[k] = __builtin_amdgcn_readlane(upto, PLAN_WAVES - 1);
    v.at[k] += __builtin_amdgcn_readlane(upto - x, wave);
  }
  return v;
}
__device__ __forceinline__ int block_scan(int v, int (*wave_sums)[PLAN_WAVES], int& all) {
  Sums<1> sum;
  v = block_scan(Sums<1>{{v}}, wave_sums, sum).at[0];
  all = sum.at[0];
  return v;
}

// ------------------------------------------------------------------ append
// What the plan tells the copying launch about an entry: rows pos .. pos + n - 1 of slot are new; page `from`, if any, held the
// first pos % page_rows rows of the page that row pos stands in now.
struct Entry { int32_t slot, pos, n, from; };
struct AppendWs { Entry* entry; int32_t *upto, *taken; };       // [B], [B] pages wanted by the entries up to this one, [P]

// What the arrays say of an entry, and what the call makes of it: pages that it keeps, and holds when all its rows are there.
struct Asked { int slot, len, pos, n; };
__device__ __forceinline__ Asked asked_of(const PagedAppendArgs& a, int b) {
  Asked x;
  x.slot = paged_slot(a.c, a.slots, b);
  x.pos = a.pos ? a.pos[b] : INT32_MAX;
  x.n = a.n_new ? a.n_new[b] : a.M;
  x.len = a.c.lens[max(x.slot, 0)];
  return x;
}
struct Want { int slot, len, pos, n, keep, pages; bool room; };
__device__ __forceinline__ Want want_of(const PagedAppendArgs& a, const Asked& x) {
  Want w;
  w.slot = x.slot;
  w.len = w.slot < 0 ? 0 : paged_clamped(x.len, a.c.W, a.c.shift);
  w.pos = min(max(x.pos, 0), w.len);
  w.n = w.slot < 0 ? 0 : min(max(x.n, 0), a.M);
  w.room = (int64_t)w.pos + w.n <= (int64_t)a.c.W << a.c.shift;
  w.keep = paged_pages(w.pos, a.c.shift);
  w.pages = w.room ? paged_pages(w.pos + w.n, a.c.shift) : w.keep;
  return w;
}
// the page that an entry's first row joins, -1 if it begins one, -2 if the table names none (the rows go into a fresh one)
__device__ __forceinline__ bool joins_page(const PagedAppendArgs& a, const Want& w) { return w.n > 0 && w.room && (w.pos & ((1 << a.c.shift) - 1)); }
__device__ __forceinline__ int page_before(const PagedAppendArgs& a, const Want& w) {        // (read whether it joins or not)
  return a.c.table[(int64_t)max(w.slot, 0) * a.c.W + max(w.keep - 1, 0)];
}

// f(x, y, i) for every i in [lo, hi), with the lane's x and y: by the lane where they are few, by the wave together where they are many
template <class F> __device__ __forceinline__ void each_page(int lo, int hi, int x, int y, F&& f) {
  const bool many = hi - lo > 4;
  if (!many)
    for (int i = lo; i < hi; ++i) f(x, y, i);
  for (unsigned long long left = __ballot(many); left; left &= left - 1) {
    const int l = __ffsll((long long)left) - 1;
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
    const int to = of(hi), xl = of(x), yl = of(y);
    for (int i = of(lo) + (int)(threadIdx.x & 63); i < to; i += 64) f(xl, yl, i);
  }
}

constexpr int LOOK = 16;                   // counts that a thread looks at in one trip to memory
constexpr int NEAR = 4096;                 // taken pages that LDS holds

// One workgroup, bound by its trips to memory one behind the other: releases, the pages that every entry wants, the lowest free
// ones, handed out in order.  64 entries of 5 rows over some 15000 pages: 7.5 us, a launch's 2 and four trips (slots, lengths,
// table, counts).
__global__ __launch_bounds__(PLAN) void paged_append_plan_kernel(PagedAppendArgs a, AppendWs ws) {
  __shared__ int owner[PAGED_MAX_BATCH];
  __shared__ int taken[NEAR];
  __shared__ int wave_sums[2][PLAN_WAVES];
  __shared__ int lacking;
  const int tid = threadIdx.x, in_page = (1 << a.c.shift) - 1;
  const bool one = a.B <= PLAN;            // every thread has at most one entry, and keeps it
  for (int s = tid; s < a.c.N; s += PLAN) owner[s] = INT32_MAX;
  if (tid == 0) lacking = 0;
  Asked asked{-1, 0, 0, 0};
  if (one && tid < a.B) asked = asked_of(a, tid);
  __syncthreads();
  for (int b = tid; b < a.B; b += PLAN) {  // the slot's first entry counts
    const int s = one ? asked.slot : paged_slot(a.c, a.slots, b);
    if (s >= 0) atomicMin(&owner[s], b);
  }
  Want w = want_of(a, asked);
  int before = one ? page_before(a, w) : -1;                    // (on the way meanwhile)
  __syncthreads();
  auto entry_at = [&](int b) {
    asked = Asked{-1, 0, 0, 0};
    if (b < a.B) asked = asked_of(a, b);
    if (asked.slot >= 0 && owner[asked.slot] != b) asked.slot = -1;
    w = want_of(a, asked);
  };
  // pages behind the kept rows are given up; of the page that is kept in part, whether there is one
  int part = -1;
  for (int b0 = 0; b0 < a.B; b0 += PLAN) {
    const int b = b0 + tid;
    if (!one) {
      entry_at(b);
      before = page_before(a, w);
    } else if (w.slot >= 0 && owner[w.slot] != b) {
      asked.slot = -1;
      w = want_of(a, asked);
    }
    part = joins_page(a, w) ? is_page(a.c, before) ? before : -2 : -1;
    each_page(w.keep, paged_pages(w.len, a.c.shift), w.slot, 0, [&](int slot, int, int i) {
      const int p = a.c.table[(int64_t)slot * a.c.W + i];
      if (is_page(a.c, p)) add_count(a.c.refs + p, -1);
    });
    if (!one && b < a.B) ws.entry[b] = Entry{w.slot, part, 0, 0};         // (looked at again below)
  }
  settle();
  // Pages wanted; a page that is kept in part and shared is copied into one of its own.  The first counts are looked at on the way.
  const bool vec = (((uintptr_t)a.c.refs) & 15) == 0;
  int held[LOOK];
  auto look = [&](int64_t p0) {
    const int64_t p = p0 + (int64_t)LOOK * tid;
    if (vec && p + LOOK <= a.c.P) {
#pragma unroll
      for (int i = 0; i < LOOK; i += 4) {
        const int4 x = *(const int4*)(a.c.refs + p + i);
        held[i] = x.x; held[i + 1] = x.y; held[i + 2] = x.z; held[i + 3] = x.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < LOOK; ++i) held[i] = p + i < a.c.P ? a.c.refs[p + i] : 1;
    }
  };
  auto count_free = [&]() {
    int n = 0;
#pragma unroll
    for (int i = 0; i < LOOK; ++i) n += held[i] <= 0;
    return n;
  };
  look(0);
  int wanted = 0, upto = 0, free0 = 0, all0 = 0;         // free pages among the first counts: of the threads up to this one, of all
  Sums<2> sums{};
  Entry e{-1, 0, 0, -1};
  for (int b0 = 0; b0 < a.B; b0 += PLAN) {
    const int b = b0 + tid;
    if (!one) {
      entry_at(b);
      part = b < a.B ? ws.entry[b].pos : -1;
    }
    int from = -1;
    if (part != -1) from = part == -2 ? -2 : a.c.refs[part] > 1 ? part : -1;
    const int need = w.pages - w.keep + (from != -1);
    if (b < a.B && !w.room) atomicAdd(&lacking, (int)(((int64_t)w.pos + w.n - ((int64_t)a.c.W << a.c.shift) + in_page) >> a.c.shift));
    e = Entry{w.slot, w.pos, w.room ? w.n : 0, from};
    const Sums<2> v = block_scan(Sums<2>{{need, b0 ? 0 : count_free()}}, wave_sums, sums);
    if (!b0) { free0 = v.at[1]; all0 = sums.at[1]; }
    upto = wanted + v.at[0];
    wanted += sums.at[0];
    if (b < a.B) { ws.entry[b] = e; ws.upto[b] = upto; }
  }
  // the lowest free pages
  int found = 0;
  for (int64_t p0 = 0; p0 < a.c.P && found < wanted; p0 += LOOK * PLAN) {
    int all = all0, at = free0;
    if (p0) {
      look(p0);
      at = block_scan(count_free(), wave_sums, all);
    }
    at += found - count_free();
#pragma unroll
    for (int i = 0; i < LOOK; ++i)
      if (held[i] <= 0) {
        if (at < NEAR) taken[at] = (int)(p0 + (int64_t)LOOK * tid + i); else ws.taken[at] = (int32_t)(p0 + (int64_t)LOOK * tid + i);
        ++at;
      }
    found += all;
  }
  if (wanted > NEAR || !one) settle(); else __syncthreads();
  if (tid == 0 && a.short_pages) a.short_pages[0] = max(wanted - found, 0) + lacking;
  for (int b0 = 0; b0 < a.B; b0 += PLAN) {
    const int b = b0 + tid;
    if (!one) {
      e = Entry{-1, 0, 0, -1};
      if (b < a.B) { e = ws.entry[b]; upto = ws.upto[b]; }
    }
    const int keep = paged_pages(e.pos, a.c.shift), own = e.from != -1;
    const int need = e.slot < 0 ? 0 : paged_pages(e.pos + e.n, a.c.shift) - keep + own;
    const bool fits = need == 0 || upto <= found;               // else the entry keeps its first rows
    const int first = upto - need;                              // of its pages among those taken
    each_page(keep - own, keep - own + (fits ? need : 0), e.slot, first - (keep - own), [&](int slot, int shifted, int i) {
      const int at = shifted + i, p = at < NEAR ? taken[at] : ws.taken[at];
      a.c.table[(int64_t)slot * a.c.W + i] = p;
      __hip_atomic_store(a.c.refs + p, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    if (e.slot >= 0) {
      if (!fits) { ws.entry[b].n = 0; ws.entry[b].from = -1; }
      else if (e.from >= 0) add_count(a.c.refs + e.from, -1);
      a.c.lens[e.slot] = fits ? e.pos + e.n : e.pos;
    }
  }
}

constexpr int STORE_ROWS = 4;              // rows of a workgroup of the copying launch

// New rows (blockIdx.x < new_blocks) and the kept rows of copied pages.  K rows are rotated on the way: the angles of a workgroup's rows
// are evaluated once, in LDS, and serve all heads.
template <bool BF16>
__global__ __launch_bounds__(256) void paged_append_store_kernel(PagedAppendArgs a, AppendWs ws, int new_blocks) {
  constexpr int E = BF16 ? 2 : 4, PIECE = BF16 ? 8 : 2;        // bytes and values of a thread's access
  __shared__ float2 cs[STORE_ROWS][64];
  const int b = blockIdx.y, tid = threadIdx.x, in_page = (1 << a.c.shift) - 1;
  const Entry e = ws.entry[b];
  const bool fresh = (int)blockIdx.x < new_blocks;
  const int r0 = fresh ? blockIdx.x * STORE_ROWS : 0, rows = fresh ? e.n : e.from >= 0 ? e.pos & in_page : 0;
  if (r0 >= rows) return;
  const int64_t row_bytes = (int64_t)a.G * a.d * E;
  const int32_t* table = a.c.table + (int64_t)e.slot * a.c.W;
  if (!fresh) {
    const int64_t to = ((int64_t)table[e.pos >> a.c.shift] << a.c.shift) * row_bytes, from = ((int64_t)e.from << a.c.shift) * row_bytes;
    constexpr int64_t piece = 256 * 16;
    const int64_t step = (int64_t)(gridDim.x - new_blocks) * piece;
    for (int64_t i = (int64_t)(blockIdx.x - new_blocks) * piece + tid * 16; i < rows * row_bytes; i += step) {
      *(u32x4*)((char*)a.c.k + to + i) = *(const u32x4*)((const char*)a.c.k + from + i);
      *(u32x4*)((char*)a.c.v + to + i) = *(const u32x4*)((const char*)a.c.v + from + i);
    }
    return;
  }
  const int here = min(STORE_ROWS, rows - r0);
  const int half = a.d >> 1;
  if (a.rope) {
    for (int i = tid; i < here * 64; i += 256) {
      const int r = i >> 6, c = i & 63;
      if (c < half) cs[r][c] = rope_cos_sin(a.rope_pos ? a.rope_pos[(int64_t)b * a.M + r0 + r] : e.pos + r0 + r, c, a.d, a.l2base);
    }
    __syncthreads();
  }
  typedef unsigned int piece_t __attribute__((ext_vector_type(PIECE * E / 4)));
  const int per_head = half / PIECE, per_row = a.G * per_head;   // (d is a multiple of 4; bf16: 128)
  for (int i = tid; i < here * per_row; i += 256) {
    const int r = i / per_row, head = i % per_row / per_head, c = i % per_head * PIECE;
    const int row = e.pos + r0 + r;
    const int64_t src = ((int64_t)b * a.M + r0 + r) * row_bytes + ((int64_t)head * a.d + c) * E;
    const int64_t dst = (((int64_t)table[row >> a.c.shift] << a.c.shift) + (row & in_page)) * row_bytes + ((int64_t)head * a.d + c) * E;
    piece_t x = *(const piece_t*)((const char*)a.k_new + src), y = *(const piece_t*)((const char*)a.k_new + src + half * E);
    const piece_t v0 = *(const piece_t*)((const char*)a.v_new + src), v1 = *(const piece_t*)((const char*)a.v_new + src + half * E);
    if (a.rope) {
      if constexpr (BF16) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 t = cs[r][c + 2 * j], u = cs[r][c + 2 * j + 1];
          const float x0 = __uint_as_float(x[j] << 16), x1 = __uint_as_float(x[j] & 0xffff0000u);
          const float y0 = __uint_as_float(y[j] << 16), y1 = __uint_as_float(y[j] & 0xffff0000u);
          x[j] = pack_bf16x2(x0 * t.x - y0 * t.y, x1 * u.x - y1 * u.y);
          y[j] = pack_bf16x2(y0 * t.x + x0 * t.y, y1 * u.x + x1 * u.y);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 t = cs[r][c + j];
          const float x0 = __uint_as_float(x[j]), y0 = __uint_as_float(y[j]);
          x[j] = __float_as_uint(x0 * t.x - y0 * t.y);
          y[j] = __float_as_uint(y0 * t.x + x0 * t.y);
        }
      }
    }
    *(piece_t*)((char*)a.c.k + dst) = x;
    *(piece_t*)((char*)a.c.k + dst + half * E) = y;
    *(piece_t*)((char*)a.c.v + dst) = v0;
    *(piece_t*)((char*)a.c.v + dst + half * E) = v1;
  }
}

// ------------------------------------------------------------------ fork
// Sources are read in one launch and targets changed in the next: a slot may be both.
struct ForkWs { int32_t *rows, *pages; };  // [B] rows that the target takes (-1: the entry does not count), [B, W] their pages

__global__ __launch_bounds__(256) void paged_fork_read_kernel(PagedCache c, const int32_t* dst, const int32_t* src, const int32_t* rows, ForkWs ws) {
  __shared__ int again;
  const int b = blockIdx.x, tid = threadIdx.x, to = dst[b], from = src[b];
  if (tid == 0) again = 0;
  __syncthreads();
  if ((unsigned)to < (unsigned)c.N)
    for (int i = tid; i < b; i += 256)
      if (dst[i] == to) again = 1;         // the target's first entry counts
  __syncthreads();
  const bool counts = (unsigned)to < (unsigned)c.N && !again;
  const int slot = (unsigned)from < (unsigned)c.N ? from : -1, len = paged_len(c, slot);
  const int n = rows ? min(max(rows[b], 0), len) : len;
  if (tid == 0) ws.rows[b] = counts ? n : -1;
  if (!counts) return;
  for (int i = tid; i < paged_pages(n, c.shift); i += 256) ws.pages[(int64_t)b * c.W + i] = c.table[(int64_t)slot * c.W + i];
}

__global__ __launch_bounds__(256) void paged_fork_write_kernel(PagedCache c, const int32_t* dst, ForkWs ws) {
  const int b = blockIdx.x, tid = threadIdx.x, n = ws.rows[b];
  if (n < 0) return;
  const int to = dst[b], had = paged_pages(paged_len(c, to), c.shift), has = paged_pages(n, c.shift);
  int32_t* row = c.table + (int64_t)to * c.W;
  for (int i = tid; i < c.W; i += 256) {
    const int old = i < had ? row[i] : -1, now = i < has ? ws.pages[(int64_t)b * c.W + i] : -1;
    row[i] = now;
    if (old == now) continue;
    if (is_page(c, old)) add_count(c.refs + old, -1);
    if (is_page(c, now)) add_count(c.refs + now, 1);
  }
  __syncthreads();                         // (everyone has read the old length)
  if (tid == 0) c.lens[to] = n;
}

// The same by one workgroup in one launch where its registers hold all pages, old and new: 24 sequences of up to 3000 rows take 5 to 7 us
// either way, but a launch takes the host 3.3 us and is the longer of the two (a pass 14.0 us with two, 11.3 with one).
constexpr int FORK_EACH = 8;               // table entries of a thread
constexpr int FORK_NEAR_ENTRIES = 256;
__global__ __launch_bounds__(PLAN) void paged_fork_kernel(PagedCache c, const int32_t* dst, const int32_t* src, const int32_t* rows, int B) {
  __shared__ int to[FORK_NEAR_ENTRIES], from[FORK_NEAR_ENTRIES], had[FORK_NEAR_ENTRIES], has[FORK_NEAR_ENTRIES];
  const int tid = threadIdx.x;
  int n = 0, mine = -1;
  if (tid < B) {
    const int s = src[tid], slot = (unsigned)s < (unsigned)c.N ? s : -1, want = rows ? rows[tid] : INT32_MAX;
    mine = dst[tid];
    const bool in = (unsigned)mine < (unsigned)c.N;
    const int len = c.lens[max(slot, 0)], old = c.lens[in ? mine : 0];
    n = slot < 0 ? 0 : min(max(want, 0), paged_clamped(len, c.W, c.shift));
    to[tid] = mine = in ? mine : -1;
    from[tid] = max(slot, 0);
    had[tid] = paged_pages(paged_clamped(old, c.W, c.shift), c.shift);
    has[tid] = paged_pages(n, c.shift);
  }
  __syncthreads();
  for (int i = 0; i < min(tid, B); ++i)
    if (to[i] == mine) mine = -1;          // the target's first entry counts
  int old[FORK_EACH], now[FORK_EACH];
#pragma unroll
  for (int e = 0; e < FORK_EACH; ++e) {
    const int at = tid + e * PLAN, b = min(at / c.W, B - 1), i = at - at / c.W * c.W;
    now[e] = c.table[(int64_t)from[b] * c.W + i];
    old[e] = c.table[(int64_t)max(to[b], 0) * c.W + i];
    if (i >= has[b]) now[e] = -1;
    if (i >= had[b]) old[e] = -1;
  }
  all_done();                              // (everything has been read)
  if (tid < B) to[tid] = mine;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < FORK_EACH; ++e) {
    const int at = tid + e * PLAN, b = at / c.W;
    if (b >= B || to[b] < 0) continue;
    c.table[(int64_t)to[b] * c.W + at - b * c.W] = now[e];
    if (old[e] == now[e]) continue;
    if (is_page(c, old[e])) add_count(c.refs + old[e], -1);
    if (is_page(c, now[e])) add_count(c.refs + now[e], 1);
  }
  if (tid < B && mine >= 0) c.lens[mine] = n;
}

// ------------------------------------------------------------------ compact
struct CompactWs { int32_t *number, *live, *count; };   // [P] new number of a live page, [P] live pages in order, [1] how many move

// Workgroup 0 numbers the live pages; the others clear the target's counts.
__global__ __launch_bounds__(PLAN) void paged_number_kernel(PagedCache from, PagedCache into, int32_t* short_pages, CompactWs ws) {
  __shared__ int wave_sums[1][PLAN_WAVES];
  const int tid = threadIdx.x;
  if (blockIdx.x) {
    for (int64_t p = (int64_t)(blockIdx.x - 1) * PLAN + tid; p < into.P; p += (int64_t)(gridDim.x - 1) * PLAN) into.refs[p] = 0;
    return;
  }
  int found = 0;
  for (int64_t p0 = 0; p0 < from.P; p0 += 4 * PLAN) {
    const int64_t p = p0 + 4 * tid;
    int n = 0, held[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      held[i] = p + i < from.P && from.refs[p + i] > 0;
      n += held[i];
    }
    int all, at = block_scan(n, wave_sums, all) - n + found;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p + i < from.P) {
        ws.number[p + i] = held[i] ? at : -1;
        if (held[i]) ws.live[at++] = (int32_t)(p + i);
      }
    found += all;
  }
  if (tid == 0) {
    ws.count[0] = min(found, into.P);
    if (short_pages) short_pages[0] = max(found - into.P, 0);
  }
}

// Workgroups 0 .. N - 1 rewrite a slot's table (its rows end before the first page that did not move); the others copy pages.
__global__ __launch_bounds__(256) void paged_move_kernel(PagedCache from, PagedCache into, int64_t page_bytes, CompactWs ws) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < from.N) {
    __shared__ int stop;
    const int s = blockIdx.x, len = paged_len(from, s), pages = paged_pages(len, from.shift);
    if (tid == 0) stop = min(pages, into.W);
    __syncthreads();
    auto number = [&](int i) {
      const int p = from.table[(int64_t)s * from.W + i], q = is_page(from, p) ? ws.number[p] : -1;
      return (unsigned)q < (unsigned)into.P ? q : -1;
    };
    for (int i = tid; i < pages; i += 256)
      if (number(i) < 0) atomicMin(&stop, i);
    __syncthreads();
    for (int i = tid; i < into.W; i += 256) {
      const int q = i < stop ? number(i) : -1;
      into.table[(int64_t)s * into.W + i] = q;
      if (q >= 0) add_count(into.refs + q, 1);
    }
    if (tid == 0) into.lens[s] = min((int64_t)len, (int64_t)stop << from.shift);
    return;
  }
  const int64_t pieces = page_bytes / 16, all = 2 * pieces * ws.count[0], step = (int64_t)(gridDim.x - from.N) * 256;
  for (int64_t i = (int64_t)(blockIdx.x - from.N) * 256 + tid; i < all; i += step) {
    const int64_t unit = i / pieces, piece = i - unit * pieces, to = unit >> 1;
    const int64_t src = (int64_t)ws.live[to] * pieces + piece, dst = to * pieces + piece;
    if (unit & 1) ((u32x4*)into.v)[dst] = ((const u32x4*)from.v)[src];
    else ((u32x4*)into.k)[dst] = ((const u32x4*)from.k)[src];
  }
}

// The same in one launch for a small pool: every workgroup numbers the live pages for itself, the first one has the tables
// and counts to itself, the others copy.  8 MB in 6.1 us instead of 6.7 (both measured together; now 5.6), a pass in 9.7 instead of 13.0 (the host's
// launches are the longer).
constexpr int COMPACT_NEAR = 4096, COMPACT_NEAR_ENTRIES = 16384;
constexpr int64_t COMPACT_NEAR_BYTES = 32 << 20;          // of K; a large pool is copied better by small workgroups
__global__ __launch_bounds__(PLAN) void paged_compact_kernel(PagedCache from, PagedCache into, int64_t page_bytes, int32_t* short_pages) {
  __shared__ int number[COMPACT_NEAR], live[COMPACT_NEAR];
  __shared__ int wave_sums[1][PLAN_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int EACH = COMPACT_NEAR / PLAN;
  int n = 0, held[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int p = EACH * tid + i;
    held[i] = p < from.P && from.refs[min(p, from.P - 1)] > 0;
    n += held[i];
  }
  int len0 = 0, p0 = 0;                    // of the wave's first slot: on the way meanwhile
  if (blockIdx.x == 0) {
    for (int p = tid; p < into.P; p += PLAN) into.refs[p] = 0;
    const int s = min(wave, from.N - 1);
    len0 = from.lens[s];
    p0 = from.table[(int64_t)s * from.W + min(lane, from.W - 1)];
  }
  int all, at = block_scan(n, wave_sums, all) - n;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    number[EACH * tid + i] = held[i] ? at : -1;
    if (held[i]) live[at++] = EACH * tid + i;
  }
  const int moved = min(all, into.P);
  if (blockIdx.x == 0) {
    settle();
    if (tid == 0 && short_pages) short_pages[0] = max(all - into.P, 0);
    for (int s = wave; s < from.N; s += PLAN_WAVES) {
      const int len = paged_clamped(s == wave ? len0 : from.lens[s], from.W, from.shift), pages = min(paged_pages(len, from.shift), into.W);
      int stop = pages;                    // the first page that did not move, once it is met
      for (int i0 = 0; i0 < into.W; i0 += 64) {
        const int i = i0 + lane;
        int p = p0;
        if (s != wave || i0) p = from.table[(int64_t)s * from.W + min(i, from.W - 1)];
        const int q = i < stop && is_page(from, p) ? number[p] : -1;
        const unsigned long long lost = __ballot(i < stop && (unsigned)q >= (unsigned)moved);
        if (lost) stop = i0 + __ffsll((long long)lost) - 1;
        if (i >= into.W) continue;
        into.table[(int64_t)s * into.W + i] = i < stop ? q : -1;
        if (i < stop) add_count(into.refs + q, 1);
      }
      if (lane == 0) into.lens[s] = min((int64_t)len, (int64_t)stop << from.shift);
    }
    return;
  }
  __syncthreads();
  const int64_t pieces = page_bytes / 16;
  for (int64_t u = blockIdx.x - 1; u < 2 * (int64_t)moved; u += gridDim.x - 1) {       // K or V of a page
    const int to = (int)(u >> 1);
    const u32x4* src = (const u32x4*)(u & 1 ? from.v : from.k) + live[to] * pieces;
    u32x4* dst = (u32x4*)(u & 1 ? into.v : into.k) + to * pieces;
    for (int64_t i = tid; i < pieces; i += PLAN) dst[i] = src[i];
  }
}

// where the queries of a draft step stand when the caller does not say: behind the rows that their sequence holds
__global__ __launch_bounds__(256) void paged_positions_kernel(PagedCache c, const int32_t* slots, int B, int M, int32_t* pos) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < B * M) pos[i] = paged_len(c, paged_slot(c, slots, i / M));
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t paged_append_ws_bytes(const PagedCache& c, int32_t B) {
  return up256((size_t)B * sizeof(Entry)) + up256((size_t)B * 4) + up256((size_t)c.P * 4);
}
void launch_paged_append(bool bf16, const PagedAppendArgs& a, void* ws, hipStream_t s) {
  AppendWs w;
  char* base = (char*)ws;
  w.entry = (Entry*)base; base += up256((size_t)a.B * sizeof(Entry));
  w.upto = (int32_t*)base; base += up256((size_t)a.B * 4);
  w.taken = (int32_t*)base;
  {
    ProfScope ps("paged_append_plan", s);
    hipLaunchKernelGGL(paged_append_plan_kernel, dim3(1), dim3(PLAN), 0, s, a, w);
  }
  const int new_blocks = (a.M + STORE_ROWS - 1) / STORE_ROWS;
  // Kept rows of copied pages: most entries have none, so their workgroups end at once, but starting them takes time too.  48 sequences,
  // a row each, pages of 4096 rows: 18.7 us with a workgroup for every four rows, 9.6 so (every entry with a copy: 135 / 140).
  int copy_blocks = ((1 << a.c.shift) - 1 + STORE_ROWS - 1) / STORE_ROWS;
  const int some = 4096 / a.B > 16 ? 4096 / a.B : 16;
  if (copy_blocks > some) copy_blocks = some;
  ProfScope ps("paged_append_store", s);
  const dim3 grid((unsigned)(new_blocks + copy_blocks), (unsigned)a.B);
  if (bf16) hipLaunchKernelGGL(paged_append_store_kernel<true>, grid, dim3(256), 0, s, a, w, new_blocks);
  else hipLaunchKernelGGL(paged_append_store_kernel<false>, grid, dim3(256), 0, s, a, w, new_blocks);
}

void launch_paged_positions(const PagedCache& c, const int32_t* slots, int32_t B, int32_t M, int32_t* pos, hipStream_t s) {
  ProfScope ps("paged_positions", s);
  hipLaunchKernelGGL(paged_positions_kernel, dim3((unsigned)((B * M + 255) / 256)), dim3(256), 0, s, c, slots, B, M, pos);
}

size_t paged_fork_ws_bytes(const PagedCache& c, int32_t B) { return up256((size_t)B * 4) + up256((size_t)B * c.W * 4); }
void launch_paged_fork(const PagedCache& c, const int32_t* dst, const int32_t* src, const int32_t* rows, int32_t B, void* ws,
                       hipStream_t s) {
  if (B <= FORK_NEAR_ENTRIES && (int64_t)B * c.W <= FORK_EACH * PLAN) {
    ProfScope ps("paged_fork", s);
    hipLaunchKernelGGL(paged_fork_kernel, dim3(1), dim3(PLAN), 0, s, c, dst, src, rows, B);
    return;
  }
  ForkWs w;
  w.rows = (int32_t*)ws;
  w.pages = (int32_t*)((char*)ws + up256((size_t)B * 4));
  {
    ProfScope ps("paged_fork_read", s);
    hipLaunchKernelGGL(paged_fork_read_kernel, dim3((unsigned)B), dim3(256), 0, s, c, dst, src, rows, w);
  }
  ProfScope ps("paged_fork_write", s);
  hipLaunchKernelGGL(paged_fork_write_kernel, dim3((unsigned)B), dim3(256), 0, s, c, dst, w);
}

size_t paged_compact_ws_bytes(const PagedCache& c) { return 2 * up256((size_t)c.P * 4) + 256; }
void launch_paged_compact(const PagedCache& from, const PagedCache& into, int64_t page_bytes, int32_t* short_pages, void* ws,
                          hipStream_t s) {
  if (from.P <= COMPACT_NEAR && (int64_t)from.N * (from.W + into.W) <= COMPACT_NEAR_ENTRIES && into.P <= COMPACT_NEAR_ENTRIES &&
      page_bytes * from.P <= COMPACT_NEAR_BYTES) {
    ProfScope ps("paged_compact", s);
    const int least = from.P < into.P ? from.P : into.P, blocks = 2 * least < 512 ? 2 * least : 512;
    hipLaunchKernelGGL(paged_compact_kernel, dim3((unsigned)(1 + blocks)), dim3(PLAN), 0, s, from, into, page_bytes, short_pages);
    return;
  }
  CompactWs w;
  w.number = (int32_t*)ws;
  w.live = (int32_t*)((char*)ws + up256((size_t)from.P * 4));
  w.count = (int32_t*)((char*)ws + 2 * up256((size_t)from.P * 4));
  {
    ProfScope ps("paged_number", s);
    hipLaunchKernelGGL(paged_number_kernel, dim3(1 + 64), dim3(PLAN), 0, s, from, into, short_pages, w);
  }
  ProfScope ps("paged_move", s);
  const int64_t most = 2 * (page_bytes / 16) * (from.P < into.P ? from.P : into.P);
  const int64_t blocks = (most + 255) / 256 < 2048 ? (most + 255) / 256 : 2048;
  hipLaunchKernelGGL(paged_move_kernel, dim3((unsigned)(from.N + blocks)), dim3(256), 0, s, from, into, page_bytes, w);
}

}  // namespace beagle
