// Host build of the picking of pages: a workgroup of 512 lanes, each with a stack of its own.  Between two barriers the waves run one behind the other, in an
// order that the caller names, a wave's lanes likewise from one of its exchanges to the next.  Reads cases, prints the pages picked.
//   in : n n_select lead R memory order off, then for every page its score, and its true one (of one of R query rows; the others' are lower or none)
//        order -1: the first wave first, -2: the last one first, else the seed of an order that is drawn anew at every turn
//   out: the n_select pages, or what went wrong
#include <ucontext.h>
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <iostream>
#include <random>
#include <string>
#include <vector>

#define __device__
#define __forceinline__ inline
#define BEAGLE_INLINE_LAMBDA
#define __syncthreads() host_barrier(__LINE__)

typedef uint32_t u32x4 __attribute__((vector_size(16)));
enum { RUNS, AT_BARRIER, AT_EXCHANGE, DONE };
struct Lane { ucontext_t at; std::vector<char> stack; int state, line; const char* op; uint64_t value; };
constexpr int LANES = 512, WAVE = 64;
static Lane lanes[LANES];
static ucontext_t scheduler;
static int now;                            // the lane that runs
static struct { struct { operator int() const { return now; } } x; } threadIdx;

[[noreturn]] static void wrong(const char* what) {
  std::printf("wrong: %s\n", what);
  std::fflush(stdout);
  std::exit(0);
}
static void wait(int state, const char* op, int line) {
  Lane& l = lanes[now];
  l.state = state; l.op = op; l.line = line;
  swapcontext(&l.at, &scheduler);
}
static void host_barrier(int line) { wait(AT_BARRIER, "barrier", line); }
// the values of a wave's lanes
static std::vector<uint64_t> all_of(const char* op, uint64_t v) {
  lanes[now].value = v;
  wait(AT_EXCHANGE, op, 0);
  std::vector<uint64_t> r(WAVE);
  for (int i = 0; i < WAVE; ++i) r[i] = lanes[now / WAVE * WAVE + i].value;
  wait(AT_EXCHANGE, "taken", 0);           // (nobody goes on before all have them)
  return r;
}
static int sum_upto(int v) {
  const auto a = all_of("sum", (uint32_t)v);
  uint32_t s = 0;
  for (int i = 0; i <= now % WAVE; ++i) s += (uint32_t)a[i];
  return (int)s;
}
template <class F> static uint32_t over_all(uint32_t v, F f) {
  const auto a = all_of("over all", v);
  uint32_t r = (uint32_t)a[0];
  for (int i = 1; i < WAVE; ++i) r = f(r, (uint32_t)a[i]);
  return r;
}
static unsigned long long __ballot(bool v) {
  const auto a = all_of("ballot", v);
  unsigned long long r = 0;
  for (int i = 0; i < WAVE; ++i) r |= (unsigned long long)a[i] << i;
  return r;
}
static int read_lane(int v, int l) { return (int)(uint32_t)all_of("lane", (uint32_t)v).at(l); }
#define __builtin_amdgcn_readlane read_lane
#define __builtin_amdgcn_readfirstlane(v) read_lane(v, 0)
static int __popcll(unsigned long long v) { return __builtin_popcountll(v); }
static float __uint_as_float(uint32_t v) { float f; std::memcpy(&f, &v, 4); return f; }
static uint32_t __float_as_uint(float f) { uint32_t v; std::memcpy(&v, &f, 4); return v; }
template <class T> static T atomicAdd(T* p, T v) { const T was = *p; *p += v; return was; }
template <class T> static T atomicMax(T* p, T v) { const T was = *p; if (v > was) *p = v; return was; }
template <class T> static T max(T a, T b) { return a > b ? a : b; }
template <class T> static T min(T a, T b) { return a < b ? a : b; }
static void hand_over() { host_barrier(__LINE__); }

#include "../paper_2505_24544_amd/csrc/paged_pick.h"

namespace {
using namespace beagle;
static_assert(alignof(PickShared) >= 16 && offsetof(PickShared, count) % 16 == 0, "four counts are read at a time");
constexpr int EDGE = 64;
struct Case {
  int n, n_select, lead, R, memory, order;
  Extent x;
  std::vector<uint32_t> scores;
  std::vector<float> truth;
  std::vector<int32_t> out;
};
Case c;
PickShared shared;

void lane() {
  auto truth = [&](int i, int r) {
    if (i < 0 || i >= c.n || r < 0 || r >= c.R) wrong("a page or a query row that there is none of");
    return r == i % c.R ? c.truth[i] : r % 2 ? NAN : c.truth[i] - 1.f;
  };
  uint32_t* s = c.scores.data() + EDGE;
  int32_t* out = c.out.data() + EDGE;
  if (c.memory) pick_pages<true>(shared, c.n, c.n_select, c.lead, c.R, s, c.x, out, truth);
  else pick_pages<false>(shared, c.n, c.n_select, c.lead, c.R, s, c.x, out, truth);
  lanes[now].state = DONE;
  swapcontext(&lanes[now].at, &scheduler);
}

// a wave as far as the next barrier
void run_wave(int w) {
  for (;;) {
    for (int i = w * WAVE; i < (w + 1) * WAVE; ++i)
      if (lanes[i].state == RUNS) { now = i; swapcontext(&scheduler, &lanes[i].at); }
    int at_exchange = 0;
    for (int i = w * WAVE; i < (w + 1) * WAVE; ++i) at_exchange += lanes[i].state == AT_EXCHANGE && !std::strcmp(lanes[i].op, lanes[w * WAVE].op);
    if (at_exchange == 0) return;
    if (at_exchange < WAVE) wrong("lanes of a wave meet at different places");
    for (int i = w * WAVE; i < (w + 1) * WAVE; ++i) lanes[i].state = RUNS;
  }
}

void run() {
  for (Lane& l : lanes) {
    l.stack.resize(1 << 16);
    getcontext(&l.at);
    l.at.uc_stack.ss_sp = l.stack.data(); l.at.uc_stack.ss_size = l.stack.size(); l.at.uc_link = nullptr;
    makecontext(&l.at, lane, 0);
    l.state = RUNS;
  }
  std::mt19937 rng((unsigned)c.order);
  std::vector<int> order;
  for (int w = 0; w < LANES / WAVE; ++w) order.push_back(c.order == -2 ? LANES / WAVE - 1 - w : w);
  for (;;) {
    if (c.order >= 0) std::shuffle(order.begin(), order.end(), rng);
    for (int w : order) run_wave(w);
    int done = 0;
    for (Lane& l : lanes) {
      done += l.state == DONE;
      if (l.state != lanes[0].state || (l.state == AT_BARRIER && l.line != lanes[0].line)) wrong("waves meet at different barriers");
    }
    if (done == LANES) return;
    for (Lane& l : lanes) l.state = RUNS;
  }
}
}  // namespace

int main() {
  std::string word;                        // (read as words: infinities)
  while (std::cin >> c.n >> c.n_select >> c.lead >> c.R >> c.memory >> c.order >> word) {
    c.x = Extent{std::strtof(word.c_str(), nullptr), INFINITY, -INFINITY};
    c.scores.assign(c.n + 2 * EDGE, 0x12345678u);
    c.truth.resize(c.n);
    c.out.assign(c.n_select + 2 * EDGE, -7);
    for (int i = 0; i < c.n; ++i) {
      std::cin >> word;
      const float v = std::strtof(word.c_str(), nullptr);
      c.scores[EDGE + i] = __float_as_uint(v);
      c.x.most = fmaxf(c.x.most, v);
      c.x.least = fminf(c.x.least, v == -INFINITY ? INFINITY : v);
      std::cin >> word;
      c.truth[i] = std::strtof(word.c_str(), nullptr);
    }
    std::memset(&shared, 0x5a, sizeof(shared));
    run();
    for (int i = 0; i < EDGE; ++i) {
      if (c.out[i] != -7 || c.out[EDGE + c.n_select + i] != -7) wrong("a write outside the list");
      if (c.scores[i] != 0x12345678u || c.scores[EDGE + c.n + i] != 0x12345678u) wrong("a write outside the scores");
    }
    for (int i = 0; i < c.n_select; ++i) std::printf(i ? " %d" : "%d", c.out[EDGE + i]);
    std::printf("\n");
  }
  return 0;
}
