// The pages with the largest scores of an entry and head, for the device and (in a test, with a workgroup's lanes one behind the other and its waves in
// any order) for the host, which brings stand-ins for what belongs to the device.
#pragma once
#include <math.h>
#include <stdint.h>

namespace beagle {
namespace {

constexpr int SELECT_THREADS = 512, SELECT_WAVES = SELECT_THREADS / 64;
constexpr int SELECT_LISTED = 240;         // pages in doubt that are kept in a list (times 2^24 query rows: 32 bits)

__device__ __forceinline__ float as_float(uint32_t v) { return __uint_as_float(v); }
#if defined(__HIPCC__)
template <int CONTROL> __device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, 0xf, 0xf, false);
}
// over the first n of the sixteen lanes of a row, the four rows, all lanes (in registers: steps through LDS take 60 ns each)
template <class F> __device__ __forceinline__ uint32_t over_row(uint32_t v, F f, int n = 16) {
  if (n > 1) v = f(v, moved<0xb1>(v));     // neighbours
  if (n > 2) v = f(v, moved<0x4e>(v));     // pairs
  if (n > 4) {
    v = f(v, moved<0x124>(v));             // turned by 4, by 8
    v = f(v, moved<0x128>(v));
  }
  return v;
}
template <class F> __device__ __forceinline__ uint32_t over_rows(uint32_t v, F f) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = f(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return f(b[0], b[1]);
}
template <class F> __device__ __forceinline__ uint32_t over_all(uint32_t v, F f) { return over_rows(over_row(v, f), f); }
// What this workgroup has written to memory, its waves read behind this: a barrier alone does not wait for stores, nor empty the vector cache of
// what it held before.
__device__ __forceinline__ void hand_over() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
}
#endif
struct MaxBits { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); } };
struct MaxOf { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return __float_as_uint(fmaxf(as_float(a), as_float(b))); } };
struct MinOf { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return __float_as_uint(fminf(as_float(a), as_float(b))); } };
struct SumOf { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return __float_as_uint(as_float(a) + as_float(b)); } };

// what the scores of some pages may be off by, and the least (but -infinity) and the greatest of them
struct Extent { float off, least, most; };

// larger scores have larger keys; 0 is no score's, and neither is the largest key
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

struct PickShared {
  alignas(16) uint32_t count[256];         // (four are read at a time)
  uint32_t state[2];
  int sure, listed, here, list[SELECT_LISTED];
  uint32_t best[SELECT_LISTED];
  int found[SELECT_WAVES];
  Extent x[SELECT_WAVES];
};

// Counts of a value from 0 to 255 of each of n elements (above: not counted), and which value the want-th largest has: state[0]; state[1] of the
// elements with it are among the want largest.
template <class Value>
__device__ __forceinline__ void value_of(PickShared& sh, int n, uint32_t want, Value value) {
  const int tid = threadIdx.x;
  if (tid < 256) sh.count[tid] = 0;
  __syncthreads();
#pragma unroll 1
  for (int i = tid; i < n; i += SELECT_THREADS) {
    const uint32_t v = value(i);
    if (v < 256) atomicAdd(&sh.count[v], 1u);
  }
  __syncthreads();
  if (tid < 64) {                                            // from the largest down: four to a lane
    const u32x4 c = *(const u32x4*)&sh.count[252 - 4 * tid];
    const uint32_t sum = c[0] + c[1] + c[2] + c[3];
    uint32_t before = (uint32_t)sum_upto((int)sum) - sum;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      if (before < want && want <= before + c[i]) { sh.state[0] = 252 - 4 * tid + i; sh.state[1] = want - before; }
      before += c[i];
    }
  }
  __syncthreads();
}

// The want-th largest key, eight bits at a time.  `want` becomes how many of the keys equal to it are among them.
__device__ __forceinline__ uint32_t largest_key(PickShared& sh, const uint32_t* keys, int n, uint32_t& want) {
  uint32_t prefix = 0;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    value_of(sh, n, want, [&](int i) {
      const uint32_t k = keys[i];
      return shift == 24 || k >> (shift + 8) == prefix ? k >> shift & 255 : 256u;
    });
    prefix = prefix << 8 | sh.state[0];
    want = sh.state[1];
    __syncthreads();
  }
  return prefix;
}

// An entry's and head's pages from their scores, whose extent the waves (or, in memory, the chunks' waves) have left; the scores are overwritten.
// (true_score(i, r): of page i and query row r, the same in sixteen neighbouring lanes; no number: passed over)
template <bool MEMORY, class TrueScore>
__device__ __forceinline__ void pick_pages(PickShared& sh, int n, int n_select, int lead, int R, uint32_t* scores, Extent x, int32_t* out,
                                           TrueScore true_score) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (lane == 0) sh.x[wave] = x;
  if (tid == 0) sh.sure = sh.listed = 0;
  if constexpr (MEMORY) hand_over();
  else __syncthreads();
  x = sh.x[lane % SELECT_WAVES];
  const float off = as_float(over_all(__float_as_uint(x.off), MaxBits()));
  // Where the n_select-th largest score is: in one of 256 parts between the least and the greatest, and of that part in one of 256.  (What
  // rounds here is far below off / 8.  -infinity counts to the lowest part; where all are alike, nothing is known.)
  const float least = as_float(over_all(__float_as_uint(x.least), MinOf())), most = as_float(over_all(__float_as_uint(x.most), MaxOf()));
  float low = -INFINITY, top = most;
  if (most - least > off && most - least < INFINITY) {
    auto part_of = [](float v, float base, float per) { return (uint32_t)(int)fminf(fmaxf((v - base) * per, 0.f), 255.f); };
    const float width = (most - least) * 0x1p-8f, per = 1.f / width;
    value_of(sh, n, n_select, [&](int i) { return part_of(as_float(scores[i]), least, per); });
    const uint32_t part = sh.state[0], want = sh.state[1];
    const float base = least + part * width;
    if (part > 0) low = base;
    if (part < 255) top = base + width;
    __syncthreads();
    if (width > off) {
      const float narrow = width * 0x1p-8f, finer = 1.f / narrow;
      value_of(sh, n, want, [&](int i) {
        const float v = as_float(scores[i]);
        return part_of(v, least, per) == part ? part_of(v, base, finer) : 256u;
      });
      const uint32_t k = sh.state[0];
      if (k > 0) low = base + k * narrow;
      if (k < 255) top = base + (k + 1) * narrow;
    }
  }
  top += 2.125f * off; low -= 2.125f * off;

  constexpr uint32_t PICKED = 0xffffffffu;
  auto meet = [&] { if constexpr (MEMORY) hand_over(); else __syncthreads(); };
  auto doubtful = [&](float v) { return !(v > top) && !(v < low); };
  auto list = [&](int* count, int i) {
    const int at = atomicAdd(count, 1);
    if (at < SELECT_LISTED) { sh.list[at] = i; sh.best[at] = key_of(-INFINITY); }
  };
  auto take_true_scores = [&](int listed) {                  // a page of the list and a query row to sixteen lanes
#pragma unroll 1
    for (uint32_t t = tid >> 4; t < (uint32_t)listed * R; t += SELECT_THREADS / 16) {
      const int l = (int)(t / (uint32_t)R);
      const float v = true_score(sh.list[l], (int)(t - (uint32_t)l * R));
      if ((tid & 15) == 0 && v == v) atomicMax(&sh.best[l], key_of(v));
    }
    __syncthreads();
  };
#pragma unroll 1
  for (int i = tid; i < n; i += SELECT_THREADS) {
    const float v = as_float(scores[i]);
    if (v > top) atomicAdd(&sh.sure, 1);
    if (doubtful(v)) list(&sh.listed, i);
  }
  __syncthreads();
  const int listed = sh.listed, wanted = n_select - sh.sure;      // in doubt, and how many of them are picked
  const bool all = listed == wanted;
  uint32_t last = PICKED - 1, ties = 0;                      // what is above `last` is picked, and the first `ties` of what equals it
  if (all || listed <= SELECT_LISTED) {
    if (!all) take_true_scores(listed);
#pragma unroll 1
    for (int i = tid; i < n; i += SELECT_THREADS) {
      const float v = as_float(scores[i]);
      if (all || !doubtful(v)) scores[i] = v > top || doubtful(v) ? PICKED : 0u;
    }
    if (!all) __syncthreads();                               // (every score has been read: a zero written now would pass for one)
    if (!all && tid < listed) {                              // how many of the others come before it
      const uint32_t mine = sh.best[tid];
      const int at = sh.list[tid];
      int before = 0;
#pragma unroll 1
      for (int l = 0; l < listed; ++l) before += sh.best[l] > mine || (sh.best[l] == mine && sh.list[l] < at);
      scores[at] = before < wanted ? PICKED : 0u;
    }
    meet();
  } else {
    // too many for a list: piece by piece they take their true scores, and the last key is looked for among all
    // (each piece has a count of its own: a wave may still have to read the first one)
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += SELECT_LISTED) {
      const int i = i0 + tid;
      if (tid == 0) sh.here = 0;
      __syncthreads();
      if (tid < SELECT_LISTED && i < n) {
        const float v = as_float(scores[i]);
        if (doubtful(v)) list(&sh.here, i);
        else scores[i] = v > top ? PICKED : 0u;
      }
      __syncthreads();
      const int here = sh.here;
      take_true_scores(here);
      if (tid < here) scores[sh.list[tid]] = sh.best[tid];
    }
    meet();
    ties = n_select;
    last = largest_key(sh, scores, n, ties);
  }
  int written = 0, taken = 0;                                // of the pages before: picked, and those with the last key
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += SELECT_THREADS) {
    const bool here = i0 + tid < n;
    const uint32_t k = here ? scores[i0 + tid] : 0;
    const unsigned long long gt = __ballot(here && k > last), eq = __ballot(here && k == last), lower = (1ull << lane) - 1;
    if (lane == 0) sh.found[wave] = __popcll(gt) | __popcll(eq) << 16;
    __syncthreads();
    const int found = lane < SELECT_WAVES ? sh.found[lane] : 0, level = found >> 16, upto = sum_upto(level);       // a wave to a lane
    const int more = (found & 0xffff) + min(level, max((int)ties - taken - (upto - level), 0)), sum = sum_upto(more);
    auto of = [](int v, int l) { return __builtin_amdgcn_readlane(v, l); };
    const int before = taken + of(upto - level, wave), tie = before + __popcll(eq & lower);
    const int at = written + of(sum - more, wave) + __popcll(gt & lower) + max(min(tie, (int)ties) - min(before, (int)ties), 0);
    if (here && (k > last || (k == last && tie < (int)ties)) && at < n_select) out[at] = lead + i0 + tid;     // (there are n_select of them)
    written += of(sum, SELECT_WAVES - 1);
    taken += of(upto, SELECT_WAVES - 1);
    __syncthreads();
  }
}

}  // namespace
}  // namespace beagle
