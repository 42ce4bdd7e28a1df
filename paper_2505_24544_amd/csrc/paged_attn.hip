// Attention of a few queries of each of B sequences over key/value rows that live in pages (decode time).
//
//   s_j = scale <q, k_j>,  lse = log sum_j exp s_j,  o = sum_j exp(s_j - lse) v_j   over the rows j that the query sees.
//
// Bound: HBM.  A visible row is fetched once for all queries of its kv head (they share the matrix instructions' columns),
// 4 * d * (queries of the head) operations per 4 * d bytes, far below the matrix pipe's rate.
//
// Split.  The visible rows of an entry are counted in blocks of 32.  The blocks of all entries, one behind the other, are cut into
// as many equal runs as there are workers, so sequences of any mix of lengths fill the chip alike and the host needs no lengths.  A
// worker is one workgroup for each kv head (and row block); its four waves take every fourth block of an entry and are joined
// through LDS.  An entry that one worker has to itself is finished there; of the others each worker leaves the unnormalised sum,
// the maximum and the weight of its part in the workspace, and a second launch joins them in the order of the rows.  Where workers suffice
// for it, each entry is cut for itself instead, so that no worker has two, and few short entries go to a workgroup each, in one launch.
//
// Measured (MI355X; rows of 8 kv heads, 32 query heads unless said; a graph's replays): 48 sequences of up to 4096 rows 95 us
// (462 MB, 4.9 TB/s), 4 of up to 32768 with 40 heads 357 (1974 MB, 5.5; a kernel that only reads reaches 6.0), 12 of up to 4096
// with 10 queries each under a tree 47.4, one of 777 rows of 32 kv heads 10.3.  The counters have every visible row fetched once from HBM, and
// vector and matrix instructions issue in a tenth of the waves' time (under the tree a fifth): they wait for rows, or for room to ask for more.
//
// Layout.  A wave keeps everything in registers and shares nothing until its end: S^T = K Q^T puts a query in a
// column (lane % 16) and four keys in a lane, which is at once the layout that O^T = V^T P^T wants of P^T.  V rows are
// read in 16-byte pieces of eight (float: four) channels; the channel that a lane's row of V^T stands for is free to
// choose, so the transposition is a matter of picking halves of registers.
#include "paged.h"
#include <math.h>

namespace beagle {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Workgroups that a compute unit holds at a time, and that the registers are made for.  Eight waves with 16 KB of rows on the way each keep
// memory busy; three workgroups of one tile (168 registers, some of them spilled) took 113 us where two take 95 (48
// sequences of up to 4096 rows, 8 kv heads), and more workgroups than fit, taken in turn, 108.
constexpr int RESIDENT = 2;
constexpr float LN2 = 0.69314718055994530942f;

// what rows that nobody sees are read from: their V must be a number (0 * NaN is NaN)
__device__ __align__(16) const unsigned char zero_row[1024] = {};

// Addresses that are picked from two places are whole numbers until they are read: the compiler would not know a picked pointer
// as one into global memory, and would wait for all loads wherever it needs one.
typedef uint64_t addr_t;
__device__ __forceinline__ u32x4 load16(addr_t p) { return *(const __attribute__((address_space(1))) u32x4*)p; }

// Every wave walks the entries by itself, 64 at a time: a lane's entry, its rows, and the blocks that it and the lanes before it have.
struct Entry { int slot, blocks, upto; PagedRows rows; };
__device__ __forceinline__ Entry entry_of(const PagedAttnArgs& a, int b) {
  Entry e;
  const int at = min(b, a.B - 1);
  const int nt = a.n_true ? a.n_true[at] : INT32_MAX;
  e.slot = paged_slot(a.c, a.slots, at);
  const int len = a.c.lens[max(e.slot, 0)];
  e.rows = paged_rows(min(e.slot < 0 ? 0 : paged_clamped(len, a.c.W, a.c.shift), a.bound), nt, a.window, a.sinks);
  e.blocks = b < a.B ? e.rows.blocks : 0;
  e.upto = sum_upto(e.blocks);             // (64 entries of 2^23 blocks: fits)
  return e;
}
__device__ __forceinline__ PagedSplit split_of(const PagedAttnArgs& a, const Entry& first) {
  auto last = [](int v) { return __builtin_amdgcn_readlane(v, 63); };
  auto runs_of = [&](const Entry& e, int shift) { return last(sum_upto(paged_runs(e.blocks, shift))); };
  int64_t all = last(first.upto), runs = runs_of(first, PAGED_RUN);
  for (int b0 = 64; b0 < a.B; b0 += 64) {
    const Entry e = entry_of(a, b0 + (threadIdx.x & 63));
    all += last(e.upto);
    runs += runs_of(e, PAGED_RUN);
  }
  int shift = PAGED_RUN;
  bool apart = paged_apart(all, runs, shift, a.target);
  if (!apart && a.long_runs && a.B <= 64) {
    shift = PAGED_LONG_RUN;
    runs = runs_of(first, shift);
    apart = paged_apart(all, runs, shift, a.target);
  }
  return paged_split(all, runs, shift, apart, a.target);
}

// over the four lanes that hold a column's keys
__device__ __forceinline__ float max_over_keys(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// infinities (and what is no number) as the largest numbers of their sign; as whole numbers, the negative bf16 are in reverse order
__device__ __forceinline__ uint32_t finite_bf16x2(uint32_t x) {
  typedef short i16x2 __attribute__((ext_vector_type(2)));
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const i16x2 above = __builtin_elementwise_min(__builtin_bit_cast(i16x2, x), i16x2{0x7f7f, 0x7f7f});
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, above), u16x2{0xff7f, 0xff7f}));
}

template <bool BF16, int NH> struct Shape {
  static constexpr int HDP = BF16 ? 128 : 64 * NH;      // head width, padded
  static constexpr int KROWS = BF16 ? 32 : 16;          // rows of a step
  static constexpr int KT = KROWS / 16;                 // score tiles of a step
  static constexpr int NJ = BF16 ? 4 : 4 * NH;          // 16-byte pieces of a row that a lane holds for the scores
  static constexpr int NV = BF16 ? 8 : 4;               // V rows of a step that a lane holds
  static constexpr int NA = BF16 ? 8 : 4 * NH;          // accumulator tiles
};

// the waves' shares of an entry, and with two tiles its queries: their registers go to the rows on the way
template <class S, int RT, int WAVES> struct Shared {
  float o[WAVES][16][S::HDP + 4], m[WAVES][RT * 16], l[WAVES][RT * 16];
  u32x4 q[RT > 1 ? RT : 1][RT > 1 ? S::NJ : 1][64];
};

// One entry's blocks first .. last - 1 for one kv head and row block: a wave takes every WAVES-th.
template <bool BF16, int NH, int RT, bool TREE, int WAVES>
__device__ __forceinline__ void attend_entry(const PagedAttnArgs& a, Shared<Shape<BF16, NH>, RT, WAVES>& sh, int b, int slot, const PagedRows rows,
                                             int first, int last, bool whole, int part, int head, int rb) {
  using S = Shape<BF16, NH>;
  constexpr int E = BF16 ? 2 : 4, HDP = S::HDP;              // bytes of a value; padded head width
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));            // what is made of it belongs to this entry: kept for the next one it would take registers
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
  const int rep = a.H / a.G, R = a.M * rep;
  const int64_t row_bytes = (int64_t)a.G * a.d * E;
  const addr_t kbase = (addr_t)a.c.k + (int64_t)head * a.d * E, vbase = (addr_t)a.c.v + (int64_t)head * a.d * E, zero = (addr_t)zero_row;
  const int32_t* table = a.c.table + (int64_t)max(slot, 0) * a.c.W;
  const int in_page = (1 << a.c.shift) - 1;

  // queries: column l16 of tile t is row r of this kv head's R = M * rep rows
  constexpr bool HELD = RT == 1;           // in registers, else in LDS
  u32x4 q[S::NJ];
  if (HELD || wave < RT) {
    const int r = (rb * RT + (HELD ? 0 : wave)) * 16 + l16, m = r / rep;
    const addr_t p = (addr_t)a.q + ((((int64_t)b * a.M + m) * a.H + head * rep + r % rep) * a.d) * E;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const int piece = (4 * j + g4) * 16;
      q[j] = load16(r < R && (BF16 || piece < a.d * E) ? p + piece : zero);
      if (!HELD) sh.q[wave][j][lane] = q[j];
    }
  }
  if (!HELD) __syncthreads();
  f32x4 acc[RT][S::NA];
  float mx[RT], sum[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    mx[t] = -INFINITY; sum[t] = 0.f;
#pragma unroll
    for (int c = 0; c < S::NA; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // scale * log2(e) as two numbers: its rounding would move every score alike, and lse with them
  const float c2 = a.c2, c2_low = a.c2_low;

  // ---- the steps of this wave: KROWS rows each, of every WAVES-th block
  constexpr int SUB = PAGED_BLOCK / S::KROWS;
  const int steps = last > first + wave ? (last - first - wave + WAVES - 1) / WAVES * SUB : 0;
  const int shift = a.c.shift;
  auto base_of = [&](int s) { return paged_block(rows, first + wave + s / SUB * WAVES) * PAGED_BLOCK + s % SUB * S::KROWS; };
  u32x4 k[S::KT][S::NJ];
  typedef u32x4 Values[S::NV][NH];
  Values v;
  f32x4 sc[RT][S::KT];
  float p[RT][S::KT][4];
  auto scores = [&]() BEAGLE_INLINE_LAMBDA {
    if (!HELD) asm volatile("" ::: "memory");        // (the queries are read again)
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int kt = 0; kt < S::KT; ++kt) sc[t][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) {
        u32x4 x = q[j];
        if (!HELD) x = sh.q[t][j][lane];
#pragma unroll
        for (int kt = 0; kt < S::KT; ++kt) {
          if constexpr (BF16) sc[t][kt] = mfma_bf16(k[kt][j], x, sc[t][kt]);
          else
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[t][kt] = mfma_f32(__uint_as_float(k[kt][j][e]), __uint_as_float(x[e]), sc[t][kt]);
        }
      }
    }
  };
  auto scaled = [&](float x, float less) BEAGLE_INLINE_LAMBDA { return fmaf(x, c2_low, fmaf(x, c2, -less)); };
  // running maximum and sum, probabilities
  auto probabilities = [&]() BEAGLE_INLINE_LAMBDA {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float top = sc[t][0][0];
#pragma unroll
      for (int e = 1; e < 4 * S::KT; ++e) top = fmaxf(top, sc[t][e / 4][e % 4]);
      const float most = fmaxf(mx[t], scaled(max_over_keys(top), 0.f)), safe = most == -INFINITY ? 0.f : most;
      if (__any(most > mx[t])) {           // (after the first steps seldom)
        const float shrink = exp2_fast(mx[t] - safe);
        sum[t] *= shrink;
#pragma unroll
        for (int c = 0; c < S::NA; ++c) acc[t][c] *= shrink;
        mx[t] = most;
      }
#pragma unroll
      for (int kt = 0; kt < S::KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) { p[t][kt][i] = exp2_fast(scaled(sc[t][kt][i], safe)); sum[t] += p[t][kt][i]; }
    }
  };
  // O^T += V^T P^T
  auto values = [&](const Values& v) BEAGLE_INLINE_LAMBDA {
    if constexpr (BF16) {
      // a probability as three bf16 numbers that add up to it: its 24 bits, eight in each (cut off, not rounded, so all differences are
      // exact); the matrix pipe has the time (two terms / three: 48 sequences of up to 4096 rows 94.5 / 94.9 us, under a tree 49.5 / 50.1)
      u32x4 term[3][RT];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t x = __float_as_uint(p[t][i >> 1][2 * (i & 1)]), y = __float_as_uint(p[t][i >> 1][2 * (i & 1) + 1]);
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            term[k][t][i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
            if (k == 2) break;
            x = __float_as_uint(__uint_as_float(x) - __uint_as_float(x & 0xffff0000u));
            y = __float_as_uint(__uint_as_float(y) - __uint_as_float(y & 0xffff0000u));
          }
        }
#pragma unroll
      for (int c = 0; c < 8; ++c) {       // channels 8 l16 + c
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = __builtin_amdgcn_perm(v[2 * i + 1][0][c >> 1], v[2 * i][0][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t][c] = mfma_bf16(w, term[0][t], acc[t][c]);
        // The second and third terms may be zero, and 0 * infinity is no number: there an infinity is the largest number
        // (48 sequences of up to 4096 rows 94.9 us without, 95.4 with; under a tree 50.1 / 51.1).
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = finite_bf16x2(w[i]);
#pragma unroll
        for (int k = 1; k < 3; ++k)
#pragma unroll
          for (int t = 0; t < RT; ++t) acc[t][c] = mfma_bf16(w, term[k][t], acc[t][c]);
      }
    } else {
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int c = 0; c < 4; ++c)       // channels 64 h + 4 l16 + c
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t][4 * h + c] = mfma_f32(__uint_as_float(v[i][h][c]), p[t][0][i], acc[t][4 * h + c]);
    }
  };

  // ---- a step's rows: a lane holds one K row of each tile (l16) and four V rows (4 g4 ..; one page: its rows are a multiple of four).
  // Rows that nobody sees, or whose page number is none, are read from zero_row, without a branch.
  struct Pages { int k[S::KT], v[S::KT]; };
  auto look = [&](int s) BEAGLE_INLINE_LAMBDA {
    Pages h;
    const int base = base_of(min(s, steps - 1)), last_row = max(rows.n - 1, 0);
#pragma unroll
    for (int t = 0; t < S::KT; ++t) {
      h.k[t] = table[min(base + 16 * t + l16, last_row) >> shift];
      h.v[t] = table[min(base + 16 * t + 4 * g4, last_row) >> shift];
    }
    return h;
  };
  // bit 4 t + i: row 16 t + 4 g4 + i is seen; bit 16 + t: row 16 t + l16
  struct Step { int base; uint32_t seen; bool masked; };
  auto seen_of = [&](const Pages& h, int s) BEAGLE_INLINE_LAMBDA {
    Step st;
    st.base = base_of(s);
    st.seen = ~0u;
    const bool all = paged_all_seen(rows, st.base, S::KROWS);
    if (!all) {
      st.seen = 0;
#pragma unroll
      for (int t = 0; t < S::KT; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) st.seen |= (uint32_t)paged_seen(rows, st.base + 16 * t + 4 * g4 + i) << (4 * t + i);
        st.seen |= (uint32_t)paged_seen(rows, st.base + 16 * t + l16) << (16 + t);
      }
    }
    bool bad = false;
#pragma unroll
    for (int t = 0; t < S::KT; ++t) {
      if ((unsigned)h.v[t] >= (unsigned)a.c.P) { st.seen &= ~(15u << 4 * t); bad = true; }
      if ((unsigned)h.k[t] >= (unsigned)a.c.P) { st.seen &= ~(1u << (16 + t)); bad = true; }
    }
    st.masked = __ballot(bad) != 0 || !all;
    return st;
  };
  auto request_k = [&](const Pages& h, const Step& st) BEAGLE_INLINE_LAMBDA {
#pragma unroll
    for (int t = 0; t < S::KT; ++t) {
      addr_t src = kbase + (((int64_t)h.k[t] << shift) + ((st.base + 16 * t + l16) & in_page)) * row_bytes + 16 * g4;
      if (!(st.seen >> (16 + t) & 1)) src = zero;
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) k[t][j] = load16(BF16 || (4 * j + g4) * 16 < a.d * E ? src + 64 * j : zero);
    }
  };
  auto request_v = [&](Values& v, const Pages& h, const Step& st) BEAGLE_INLINE_LAMBDA {
#pragma unroll
    for (int t = 0; t < S::KT; ++t) {
      addr_t src = vbase + (((int64_t)h.v[t] << shift) + ((st.base + 16 * t + 4 * g4) & in_page)) * row_bytes + 16 * l16;
#pragma unroll
      for (int i = 0; i < 4; ++i, src += row_bytes)
#pragma unroll
        for (int n = 0; n < NH; ++n) {
          const bool there = (st.seen >> (4 * t + i) & 1) && (BF16 || (16 * n + l16) * 16 < a.d * E);
          v[4 * t + i][n] = load16(there ? src + 256 * n : zero);
        }
    }
  };
  auto hide = [&](const Step& st) BEAGLE_INLINE_LAMBDA {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int e = 0; e < 4 * S::KT; ++e)
        if (!(st.seen >> e & 1)) sc[t][e / 4][e % 4] = -INFINITY;
  };
  // Steps of true rows: the rows of the next step travel while this one is computed, its page numbers a step further ahead.  K's registers
  // are free once the scores are there; V has a second set (4 sequences of up to 32768 rows, 40 heads: 365 us without, 355 with).
  // (Addresses of whole steps in scalar registers, and half the vector instructions with that: the registers that
  // two ways of addressing take cost 3 to 30 % instead.)
  int plain = steps;
  if constexpr (TREE)
    while (plain > 0 && base_of(plain - 1) + S::KROWS > rows.nt) --plain;
  Pages next;                              // page numbers of the step behind those requested; behind the loop those of step `plain`
  if (steps > 0) next = look(0);
  if (plain > 0) {
    Step st = seen_of(next, 0);
    request_k(next, st);
    request_v(v, next, st);
    next = look(1);
    auto step = [&](int s, Values& mine, Values& others) BEAGLE_INLINE_LAMBDA {
      scores();
      Step ahead = st;
      const Pages now = next;
      if (s + 1 < plain) {
        ahead = seen_of(now, s + 1);
        request_k(now, ahead);
        request_v(others, now, ahead);
        next = look(s + 2);
      }
      if (st.masked) hide(st);
      probabilities();
      values(mine);
      st = ahead;
    };
    Values w;
    for (int s = 0; s < plain; s += 2) {
      step(s, v, w);
      if (s + 1 < plain) step(s + 1, w, v);
    }
  }
  if constexpr (TREE)
    for (int s = plain; s < steps; ++s) {
      if (s > plain) next = look(s);
      const Step st = seen_of(next, s);
      request_k(next, st);
      request_v(v, next, st);
      scores();
      hide(st);
      // the step's rows in a query's word of bits: true ones set, drafted ones as the tree has them
      const int off = st.base - rows.nt, word = off >> 5;          // (rounds down)
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const uint32_t* row = a.tree + ((int64_t)b * a.M + min(((rb * RT + t) * 16 + l16) / rep, a.M - 1)) * a.words;
        const bool lo_in = (unsigned)word < (unsigned)a.words, hi_in = (unsigned)(word + 1) < (unsigned)a.words;
        const uint32_t lo = lo_in ? row[word] : 0, hi = hi_in ? row[word + 1] : 0;
        const uint32_t bits = (uint32_t)((((uint64_t)hi << 32) | lo) >> (off & 31)) | (off <= -32 ? ~0u : off < 0 ? (1u << -off) - 1 : 0);
#pragma unroll
        for (int e = 0; e < 4 * S::KT; ++e)
          if (!(bits >> (16 * (e / 4) + 4 * g4 + e % 4) & 1u)) sc[t][e / 4][e % 4] = -INFINITY;
      }
      probabilities();
      // A drafted row that only some queries see may hold what is no number, which the others must not meet (0 * NaN is
      // NaN).  The matrix instructions mix all rows into all queries, so such a step adds row by row where it is seen.
      unsigned top = 0;
#pragma unroll
      for (int i = 0; i < S::NV; ++i)
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const unsigned x = v[i][h][e];
            top = max(top, x & 0x7f800000u);
            if constexpr (BF16) top = max(top, (x << 16) & 0x7f800000u);
          }
      if (__ballot(top == 0x7f800000u) == 0) {
        values(v);
        continue;
      }
      float* mine = sh.o[wave][l16];             // (free until the end)
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int e = 0; e < 4 * S::KT; ++e) mine[16 * (e / 4) + 4 * g4 + e % 4] = sc[t][e / 4][e % 4] == -INFINITY ? -1.f : p[t][e / 4][e % 4];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (int j = 0; j < S::KROWS; ++j) {
          const float w = mine[j];
          const int row = st.base + j, pg = paged_page(table, row, paged_seen(rows, row), shift, a.c.P);
          if (w == -1.f || pg < 0) continue;
          const char* src = (const char*)vbase + (((int64_t)pg << shift) + (row & in_page)) * row_bytes;
#pragma unroll
          for (int c = 0; c < S::NA; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int ch = BF16 ? 8 * (4 * g4 + i) + c : 64 * (c / 4) + 4 * (4 * g4 + i) + c % 4;
              if constexpr (BF16) acc[t][c][i] += w * bf16_to_f32(((const bf16_t*)src)[ch]);
              else if (ch < a.d) acc[t][c][i] += w * ((const float*)src)[ch];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }

  // ---- the waves' shares, then the workgroup's result
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float l = sum[t];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g4 == 0) { sh.m[wave][16 * t + l16] = mx[t]; sh.l[wave][16 * t + l16] = l; }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (t) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < S::NA; c += 4) {
        // accumulator row 4 g4 + i: bf16 channels 8 (4 g4 + i) + c, float channels 64 h + 4 (4 g4 + i) + c % 4
        const int ch = BF16 ? 8 * (4 * g4 + i) + c : 16 * c + 4 * (4 * g4 + i);
        *(f32x4*)&sh.o[wave][l16][ch] = f32x4{acc[t][c][i], acc[t][c + 1][i], acc[t][c + 2][i], acc[t][c + 3][i]};
      }
    __syncthreads();
    const int col = tid >> 4, r = (rb * RT + t) * 16 + col;
    if (r >= R || col >= 16) continue;
    float m = -INFINITY, l = 0.f, w[WAVES];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) m = fmaxf(m, sh.m[i][16 * t + col]);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      w[i] = m == -INFINITY ? 0.f : exp2_fast(sh.m[i][16 * t + col] - m);
      l += sh.l[i][16 * t + col] * w[i];
    }
    const int qi = r / rep, h = head * rep + r % rep;
    const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
    const int64_t prow = ((int64_t)part * a.G + head) * R + r;      // (whole: not used)
#pragma unroll
    for (int half = 0; half < HDP / 64; ++half) {
      const int ch = 64 * half + 4 * (tid & 15);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < WAVES; ++i) o += *(const f32x4*)&sh.o[i][col][ch] * w[i];
      o *= inv;
      if (!whole) { *(f32x4*)(a.part + prow * HDP + ch) = o; continue; }
      if (ch >= a.d) continue;
      const int64_t at = (((int64_t)b * a.M + qi) * a.H + h) * a.d + ch;
      if constexpr (BF16) *(uint2*)((bf16_t*)a.o + at) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
      else *(f32x4*)((float*)a.o + at) = o;
    }
    if ((tid & 15) == 0) {
      if (whole) a.lse[((int64_t)b * a.H + h) * a.M + qi] = (m + __log2f(l)) * LN2;
      else *(float2*)(a.ml + prow * 2) = make_float2(m, l);
    }
  }
}

// BF16: head width 128.  Float: NH = 1 for widths up to 64, 2 up to 128.  RT: tiles of 16 query rows that a workgroup takes.
// TREE: rows from n_true on are seen as the tree's bits say.
// WHOLE: a workgroup of eight waves takes an entry (`worker` is its number), for few and short ones: nothing to look up, to cut or to join.
template <bool BF16, int NH, int RT, bool TREE, bool WHOLE>
__global__ __launch_bounds__(WHOLE ? 512 : 256, WHOLE ? 1 : RESIDENT) void paged_attn_kernel(PagedAttnArgs a, int rowblocks) {
  constexpr int WAVES = WHOLE ? 8 : 4;
  __shared__ Shared<Shape<BF16, NH>, RT, WAVES> shared;
  const int lane = threadIdx.x & 63;
  // row blocks of one worker and head stand eight workgroups apart: on one XCD, whose L2 has the rows after the first
  const int id = blockIdx.x, ug = id / (8 * rowblocks) * 8 + id % 8, rb = id / 8 % rowblocks;
  const int head = ug % a.G, worker = ug / a.G;
  if constexpr (WHOLE) {
    if (worker >= a.B) return;
    auto wave = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int slot = wave(paged_slot(a.c, a.slots, worker)), nt = wave(a.n_true ? a.n_true[worker] : INT32_MAX);
    const PagedRows rows = paged_rows(min(wave(paged_len(a.c, slot)), a.bound), nt, a.window, a.sinks);
    attend_entry<BF16, NH, RT, TREE, WAVES>(a, shared, worker, slot, rows, 0, rows.blocks, true, 0, head, rb);
    return;
  }
  const Entry group0 = entry_of(a, lane);
  const PagedSplit split = split_of(a, group0);
  if (worker >= split.workers) return;
  const int64_t lo = paged_cut(split, worker), hi = paged_cut(split, worker + 1);
  int64_t base0 = 0;                       // blocks before this group of entries
  bool used = false;                       // LDS holds another entry's shares
  for (int b0 = 0; b0 < a.B && base0 < hi; b0 += 64) {
    Entry e = group0;
    if (b0) e = entry_of(a, b0 + lane);
    const int counted = paged_counted(split, e.blocks), upto = split.apart ? sum_upto(counted) : e.upto;
    const int64_t start = base0 + upto - counted;
    const PagedShare share = paged_share(split, start, e.blocks, lo, hi);
    unsigned long long mine = __ballot(share.from < share.to);
    if (head == 0 && rb == 0 && threadIdx.x < 64 && share.from == 0 && share.to > 0)       // for the join: an entry's first worker, and how many have a part
      a.parts[b0 + lane] = make_int2(worker, share.to == e.blocks ? 1 : paged_worker_of(split, start + e.blocks - 1) - worker + 1);
    base0 += __builtin_amdgcn_readlane(upto, 63);
    while (mine) {
      const int l = __ffsll((long long)mine) - 1;
      mine &= mine - 1;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      const int b = b0 + l, slot = of(e.slot), first = of(share.from), last = of(share.to);
      const PagedRows rows = paged_rows(of(e.rows.n), of(e.rows.nt), a.window, a.sinks);
      const bool whole = last - first == rows.blocks;
      if (used) __syncthreads();
      used = true;
      // a part's sums: one place for the entry that the worker goes on with, one for the entry that it begins
      attend_entry<BF16, NH, RT, TREE, WAVES>(a, shared, b, slot, rows, first, last, whole, 2 * worker + (first == 0), head, rb);
    }
  }
}

// The parts of an entry, in order.  A row is joined by 32 (narrow floats: 16) lanes; ROWS of them share a workgroup, whose other
// lanes take every (groups / ROWS)-th part of a row each and meet in LDS.
template <bool BF16, int HDP, int ROWS>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int LANES = HDP / 4, GROUPS = 256 / LANES, SPLIT = GROUPS / ROWS;
  __shared__ float so[GROUPS][HDP];
  __shared__ float sm[GROUPS], sl[GROUPS];
  const int rep = a.H / a.G, R = a.M * rep;
  const int b = blockIdx.y;
  const int2 from = a.parts[b];
  const int w0 = min(max(from.x, 0), a.target - 1), shares = min(from.y, a.target - w0);
  if (shares <= 1) return;
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
  if (n < a.G * R) {
    const int64_t row0 = ((int64_t)2 * w0 * a.G + head) * R + r, step = (int64_t)a.G * R;
    constexpr int AT_ONCE = 4;
    for (int i = group % SPLIT; i < shares; i += SPLIT * AT_ONCE) {
      float2 ml[AT_ONCE];
      f32x4 po[AT_ONCE];
#pragma unroll
      for (int e = 0; e < AT_ONCE; ++e) {
        const int n = min(i + e * SPLIT, shares - 1);
        const int64_t row = row0 + step * (n ? 2 * n : 1);
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

// An entry goes whole to a workgroup for each head if there are at most WHOLE_GROUPS of them (a compute unit each) and it has at most two
// blocks for each of the eight waves, one if a wave reads a block in two steps of more than 64 floats; or, in bf16, no more blocks than a quarter of
// the workgroups: then the cut calls are bound by the memory's rate and these, without a second launch, reach as much.
// A workgroup of its own / cut and joined, us (bf16, 1 query, rows in the caches of a graph's replays): 1 sequence of 8 heads, 400 rows 9.3 / 10.1, 700
// 11.9 / 10.0; 8 sequences of 32 heads, 1000 rows 24.0 / 27.5, 2000 42.3 / 46.1 (uneven lengths 33.8 / 34.3); 20 of 4 heads of 128 floats, 400 rows
// 20.9 / 19.3.
constexpr int WHOLE_GROUPS = 256;
int whole_blocks(bool bf16, int d, int64_t groups) {
  if (!bf16) return d <= 64 ? 16 : 8;
  return groups / 4 > 16 ? (int)(groups / 4) : 16;
}
constexpr int MAX_TILES = 2;               // of 16 query rows that a workgroup takes
struct Tiles { int each, blocks; };        // tiles of a workgroup, workgroups that the rows of a kv head take
Tiles tiles_of(int R) {
  const int all = (R + 15) / 16, blocks = (all + MAX_TILES - 1) / MAX_TILES;
  return {(all + blocks - 1) / blocks, blocks};
}
// workers of a kv head and row block: the compute units hold them all at once
int workers_aimed(int R, int G) {
  const int64_t per = (int64_t)G * tiles_of(R).blocks, slots = 256 * RESIDENT;
  return per < slots ? (int)(slots / per) : 1;
}

// rows of sums of parts: a worker has at most two entries in part (see paged_index.h), and one that is alone none
int64_t part_rows(int R, int G) {
  const int workers = workers_aimed(R, G);
  return workers > 1 ? (int64_t)2 * workers * G * R : 0;
}

}  // namespace

// The parts, and for each entry who has them.
size_t paged_attn_ws_bytes(int32_t B, int32_t M, int32_t H, int32_t G) {
  return (size_t)part_rows(M * (H / G), G) * (128 + 2) * sizeof(float) + (size_t)B * sizeof(int2);
}

void launch_paged_attn(bool bf16, PagedAttnArgs a, void* ws, hipStream_t s) {
  const int R = a.M * (a.H / a.G);
  const Tiles tiles = tiles_of(R);
  // blocks that an entry can have: those of the longest sequence, or of the window's and the first rows (their edges not counted as whole)
  int64_t most = (a.bound + PAGED_BLOCK - 1) / PAGED_BLOCK;
  if (a.window > 0 && !a.n_true) {
    const int64_t seen = (int64_t)(a.window / PAGED_BLOCK) + a.sinks / PAGED_BLOCK + 4;
    if (seen < most) most = seen;
  }
  const int64_t groups = (int64_t)a.B * a.G * tiles.blocks;
  const bool whole = groups <= WHOLE_GROUPS && most <= whole_blocks(bf16, a.d, groups);
  a.target = workers_aimed(R, a.G);
  a.long_runs = bf16;                      // (floats: what a block costs is its products, and more workers take less)
  // both parts above zero: a hidden row's score is -infinity and has to stay it
  const double c2 = fmax(a.scale * 1.44269504088896340736, 2e-38);
  a.c2 = (float)c2;
  if ((double)a.c2 >= c2) a.c2 = nextafterf(a.c2, 0.f);
  a.c2_low = fmaxf((float)(c2 - a.c2), 1.1754944e-38f);
  const int64_t rows = part_rows(R, a.G);
  a.part = (float*)ws;
  a.ml = a.part + rows * 128;
  a.parts = (int2*)(a.ml + rows * 2);
  const int heads = (whole ? a.B : a.target) * a.G;       // of all entries or workers
  const dim3 grid((unsigned)((heads + 7) / 8 * 8 * tiles.blocks)), wg(whole ? 512 : 256);
  const bool tree = a.n_true != nullptr, narrow = !bf16 && a.d <= 64;
  {
    ProfScope ps("paged_attn", s);
    auto go = [&](auto bf_, auto nh_, auto rt_, auto whole_) {
      constexpr bool BF = decltype(bf_)::value != 0, WH = decltype(whole_)::value != 0;
      constexpr int NH = decltype(nh_)::value, RT = decltype(rt_)::value;
      if (tree) hipLaunchKernelGGL((paged_attn_kernel<BF, NH, RT, true, WH>), grid, wg, 0, s, a, tiles.blocks);
      else hipLaunchKernelGGL((paged_attn_kernel<BF, NH, RT, false, WH>), grid, wg, 0, s, a, tiles.blocks);
    };
    auto with = [&](auto bf_, auto nh_) {
      if (tiles.each == 1 && whole) go(bf_, nh_, int_c<1>{}, int_c<1>{});
      else if (whole) go(bf_, nh_, int_c<2>{}, int_c<1>{});
      else if (tiles.each == 1) go(bf_, nh_, int_c<1>{}, int_c<0>{});
      else go(bf_, nh_, int_c<2>{}, int_c<0>{});
    };
    if (bf16) with(int_c<1>{}, int_c<1>{});
    else if (narrow) with(int_c<0>{}, int_c<1>{});
    else with(int_c<0>{}, int_c<2>{});
  }
  if (whole || a.target == 1 || most <= 1 << PAGED_RUN) return;    // no entry is cut: nothing to join
  ProfScope ps("paged_join", s);
  auto join = [&](auto bf_, auto hdp_) {
    constexpr bool BF = decltype(bf_)::value != 0;
    constexpr int HDP = decltype(hdp_)::value, MANY = 256 / (HDP / 4);
    const int64_t all = (int64_t)a.H * a.M;
    if (all * a.B <= 1024) hipLaunchKernelGGL((paged_join_kernel<BF, HDP, 1>), dim3((unsigned)all, (unsigned)a.B), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_join_kernel<BF, HDP, MANY>), dim3((unsigned)((all + MANY - 1) / MANY), (unsigned)a.B), dim3(256), 0, s, a);
  };
  if (bf16) join(int_c<1>{}, int_c<128>{});
  else if (narrow) join(int_c<0>{}, int_c<64>{});
  else join(int_c<0>{}, int_c<128>{});
}

}  // namespace beagle
