// Attention of a few queries of each of B sequences whose first rows are the same within groups of them (branches of one
// sequence, users under one prompt): the common rows are fetched once for all queries of the group, every sequence's own rows once for its own.
//
//   over rows P (common) and T (own):  m = max(m_P, m_T),  l = l_P 2^(m_P - m) + l_T 2^(m_T - m),  o = (o_P 2^(m_P - m) + o_T 2^(m_T - m)) / l
//
// Three launches.  The first, one workgroup, divides the work into units: some blocks of 32 rows for a few tiles of 16 query rows, of a
// group's common rows or of an entry's own.  The second computes units, the third joins every query row's parts in the order of the rows.
#include "paged_attend.h"

namespace beagle {
namespace {

constexpr int PLAN_THREADS = 1024;
// What a block of 32 rows costs a workgroup: common rows for one block of query rows, own rows.
constexpr int COST_COMMON = 1, COST_OWN = 2;

struct Unit {
  int32_t own, b, slot, rb;                // own rows of entry b, or a group's that begins with entry b; which block of query rows
  int32_t first, last, n, nt;              // blocks; rows in all, true ones
  int32_t from, entries;                   // own rows: from this row on; of how many entries the query rows are
  int64_t part;                            // row of the parts, per kv head
};
// where the parts of an entry's query rows are: rows [common + i * stride + ..], i < n_common, [own + i * R + ..], i < n_own
struct Where { int64_t common, own; int32_t stride, offset, n_common, n_own; };
struct Plan { int32_t units, pad[63]; };

struct SharedLayout { size_t units, where, ml, part, total; int64_t max_units, rows; };

struct Shares {
  PagedAttnArgs a;
  const int32_t *group_first, *n_shared;
  int32_t groups, workers, common_cols, own_blocks;          // query rows of a unit of common rows; blocks of query rows of an entry
  Plan* plan; Unit* units; Where* where;
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
  r.cols = r.blocks ? (int)(((int64_t)r.entries * s.a.M * (s.a.H / s.a.G) + s.common_cols - 1) / s.common_cols) : 0;
  return r;
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
  // what there is to do, and from it the blocks that a unit gets
  int64_t common = 0, own = 0, sum;
  for (int g = tid; g < s.groups; g += PLAN_THREADS) { const Group x = group_of(s, first, g); common += (int64_t)x.blocks * x.cols; }
  for (int b = tid; b < s.a.B; b += PLAN_THREADS) own += (int64_t)own_of(s, first, b).blocks * s.own_blocks;
  sum_before(common * COST_COMMON + own * COST_OWN, tmp, &sum);
  const int64_t aim = (sum + s.workers - 1) / s.workers;
  const int64_t long_common = max((aim + COST_COMMON - 1) / COST_COMMON, (int64_t)4), long_own = max((aim + COST_OWN - 1) / COST_OWN, (int64_t)4);

  int units = 0;
  int64_t parts = 0;
  for (int g0 = 0; g0 < s.groups; g0 += PLAN_THREADS) {
    const Group x = group_of(s, first, g0 + tid);
    const int cuts = x.blocks ? (int)((x.blocks + long_common - 1) / long_common) : 0;
    int64_t all;
    const int64_t at = sum_before((int64_t)cuts * x.cols, tmp, &all), row = sum_before(cuts * x.entries * R, tmp, &sum);
    base[tid] = (int)at; rows[tid] = parts + row;
    if (tid == 0) base[PLAN_THREADS] = (int)all;
    __syncthreads();
    // units of each group: cut after cut of its rows, those of a cut one behind the other
    for (int u = tid; u < (int)all; u += PLAN_THREADS) {
      const int i = group_with(base, PLAN_THREADS, u);
      const Group y = group_of(s, first, g0 + i);
      const int n = (int)((y.blocks + long_common - 1) / long_common), cut = (u - base[i]) / y.cols;
      s.units[units + u] = Unit{0, y.lo, y.slot, (u - base[i]) % y.cols, (int)((int64_t)y.blocks * cut / n), (int)((int64_t)y.blocks * (cut + 1) / n),
                                y.n, y.n, 0, y.entries, rows[i] + cut * y.entries * R};
    }
    const int last = min(g0 + PLAN_THREADS, s.groups);
    for (int b = first[g0] + tid; b < first[last]; b += PLAN_THREADS) {
      const int g = group_with(first, s.groups, b);
      const Group y = group_of(s, first, g);
      Where* w = s.where + b;
      w->common = rows[g - g0]; w->stride = (int)(y.entries * R); w->offset = (int)((b - y.lo) * R);
      w->n_common = y.blocks ? (int)((y.blocks + long_common - 1) / long_common) : 0;
    }
    units += (int)all; parts += sum;
    __syncthreads();
  }
  for (int b0 = 0; b0 < s.a.B; b0 += PLAN_THREADS) {
    const int b = b0 + tid;
    const Own x = own_of(s, first, b);
    const int cuts = (int)((x.blocks + long_own - 1) / long_own);
    int64_t all;
    const int64_t at = sum_before((int64_t)cuts * s.own_blocks, tmp, &all), row = sum_before(cuts * R, tmp, &sum);
    base[tid] = (int)at; rows[tid] = parts + row;
    if (tid == 0) base[PLAN_THREADS] = (int)all;
    __syncthreads();
    for (int u = tid; u < (int)all; u += PLAN_THREADS) {
      const int i = group_with(base, PLAN_THREADS, u);
      const Own y = own_of(s, first, b0 + i);
      const int n = (int)((y.blocks + long_own - 1) / long_own), cut = (u - base[i]) / s.own_blocks;
      s.units[units + u] = Unit{1, b0 + i, y.slot, (u - base[i]) % s.own_blocks, (int)((int64_t)y.blocks * cut / n),
                                (int)((int64_t)y.blocks * (cut + 1) / n), y.n, y.nt, y.from, 1, rows[i] + cut * R};
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

template <bool BF16, int NH, int RTC, int RTO, bool TREE>
__global__ __launch_bounds__(256, RESIDENT) void paged_shared_kernel(Shares s) {
  using S = Shape<BF16, NH>;
  __shared__ union { Shared<S, RTC, 4, PREFIX> common; Shared<S, RTO, 4, SUFFIX> own; } shared;
  const int head = blockIdx.x % s.a.G;
  auto wave = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int units = wave(s.plan->units);
  for (int u = blockIdx.x / s.a.G; u < units; u += s.workers) {
    const Unit x = s.units[u];
    const int R = s.a.M * (s.a.H / s.a.G) * wave(x.entries);
    Item item = {};
    item.R = R; item.entries = wave(x.entries);
    const int64_t part = (int64_t)wave((int)(x.part >> 32)) << 32 | (uint32_t)wave((int)x.part);
    item.part_row = part * s.a.G + (int64_t)head * R;
    const int b = wave(x.b), slot = wave(x.slot), rb = wave(x.rb), first = wave(x.first), last = wave(x.last), n = wave(x.n);
    if (u >= s.workers) __syncthreads();   // (LDS holds the unit before)
    if (wave(x.own)) attend_entry<BF16, NH, RTO, TREE, 4, SUFFIX>(s.a, shared.own, item, b, slot, paged_rows_from(n, wave(x.nt), wave(x.from)),
                                                                first, last, false, 0, head, rb);
    else attend_entry<BF16, NH, RTC, false, 4, PREFIX>(s.a, shared.common, item, b, slot, paged_rows(n, n, 0, 0), first, last, false, 0, head, rb);
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
int shared_workers(int G) { return G < 256 * RESIDENT ? 256 * RESIDENT / G : 1; }

// A unit has at least an equal share of the blocks, so that cutting adds at most `workers` units to those that groups and entries
// have uncut, and as many query rows to the parts.
SharedLayout shared_layout(int32_t B, int32_t M, int32_t H, int32_t G) {
  const int64_t R = (int64_t)M * (H / G), workers = shared_workers(G);
  const Tiles own = tiles_of((int)R);
  const int64_t cols = 16 * COMMON_TILES;
  SharedLayout l;
  l.max_units = workers + B + (B * R + cols - 1) / cols + workers + (int64_t)B * own.blocks;
  l.rows = workers * cols + B * R + workers * 16 * own.each + B * R;
  size_t at = sizeof(Plan);
  auto take = [&](size_t n) { const size_t o = at; at = (at + n + 255) / 256 * 256; return o; };
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
  x.units = (Unit*)(at + l.units);
  x.where = (Where*)(at + l.where);
  x.a.ml = (float*)(at + l.ml);
  x.a.part = (float*)(at + l.part);
  x.group_first = p.group_first; x.n_shared = p.n_shared; x.groups = p.groups;
  const Tiles own = tiles_of(p.a.M * (p.a.H / p.a.G));
  x.workers = shared_workers(p.a.G);
  x.common_cols = 16 * COMMON_TILES;
  x.own_blocks = own.blocks;
  {
    ProfScope ps("paged_shared_plan", s);
    hipLaunchKernelGGL(paged_shared_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, x);
  }
  const bool narrow = !bf16 && p.a.d <= 64, tree = p.a.n_true != nullptr;
  {
    ProfScope ps("paged_shared", s);
    const dim3 grid((unsigned)(x.workers * p.a.G));
    auto go = [&](auto bf_, auto nh_, auto rt_) {
      constexpr bool BF = decltype(bf_)::value != 0;
      constexpr int NH = decltype(nh_)::value, RT = decltype(rt_)::value;
      if (tree) hipLaunchKernelGGL((paged_shared_kernel<BF, NH, COMMON_TILES, RT, true>), grid, dim3(256), 0, s, x);
      else hipLaunchKernelGGL((paged_shared_kernel<BF, NH, COMMON_TILES, RT, false>), grid, dim3(256), 0, s, x);
    };
    auto with = [&](auto bf_, auto nh_) { own.each == 1 ? go(bf_, nh_, int_c<1>{}) : go(bf_, nh_, int_c<2>{}); };
    if (bf16) with(int_c<1>{}, int_c<1>{});
    else if (narrow) with(int_c<0>{}, int_c<1>{});
    else with(int_c<0>{}, int_c<2>{});
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
