// Attention of a few queries of each of B sequences over key/value rows that live in pages (decode time).
//
//   s_j = scale <q, k_j>,  lse = log sum_j exp s_j,  o = sum_j exp(s_j - lse) v_j   over the rows j that the query sees.
//
// Bound: HBM.  A visible row is fetched once for all queries of its kv head (they share the matrix instructions' columns),
// 4 * d * (queries of the head) operations per 4 * d bytes, far below the matrix pipe's rate.
//
// Split.  The visible rows of an entry are counted in blocks of 32; a unit is a run of blocks of one entry, as long as all
// blocks of the batch divided by the units aimed at, so sequences of any mix of lengths fill the chip alike and the host
// needs no lengths.  One workgroup takes a unit of one kv head; its four waves take every fourth block and are joined
// through LDS.  An entry of one unit is finished there; the others leave unnormalised sums, maximum and weight
// of each unit in the workspace, and a second launch joins them in the order of the rows.
//
// Layout.  A wave keeps everything in registers and shares nothing until its end: S^T = K Q^T puts a query in a
// column (lane % 16) and four keys in a lane, which is at once the layout that O^T = V^T P^T wants of P^T.  V rows are
// read in 16-byte pieces of eight (float: four) channels; the channel that a lane's row of V^T stands for is free to
// choose, so the transposition is a matter of picking halves of registers.
#include "paged.h"

namespace beagle {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int WAVES = 4;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// what rows that nobody sees are read from: their V must be a number (0 * NaN is NaN)
__device__ __align__(16) const unsigned char zero_row[1024] = {};

__device__ __forceinline__ PagedRows rows_of(const PagedAttnArgs& a, int slot, int b) {
  const int n = min(paged_len(a.c, slot), a.bound);
  return paged_rows(n, a.n_true ? a.n_true[b] : n, a.window, a.sinks);
}

// Where a unit lives: entry, its blocks, and where its partial sums go (first unit of the entry; units that the entry has).
struct Unit { int b, i, units, first, chunk; };
// Every wave walks the entries by itself, 64 at a time.  want_entry: the unit 0 of entry `which`; else unit number `which`
// (b = -1: there are fewer).
__device__ Unit find_unit(const PagedAttnArgs& a, int which, bool want_entry) {
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int b = b0 + lane;
    int blocks = b < a.B ? rows_of(a, paged_slot(a.c, a.slots, b), b).blocks : 0;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) blocks += __shfl_xor(blocks, m);       // (64 entries of 2^23 blocks: fits)
    total += __builtin_amdgcn_readfirstlane(blocks);
  }
  Unit u;
  u.chunk = paged_chunk(total, a.target, a.least);
  u.b = -1;
  int base = 0, parts = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int b = b0 + lane;
    const int mine = b < a.B ? paged_units(rows_of(a, paged_slot(a.c, a.slots, b), b).blocks, u.chunk) : 0;
    const int kept = mine > 1 ? mine : 0;
    int upto = mine, pupto = kept;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int x = __shfl_up(upto, m), y = __shfl_up(pupto, m);
      if (lane >= m) { upto += x; pupto += y; }
    }
    const bool hit = want_entry ? b == which : b < a.B && which >= base + upto - mine && which < base + upto;
    const unsigned long long at = __ballot(hit);
    if (at) {
      const int l = __ffsll((long long)at) - 1;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      u.b = b0 + l;
      u.units = of(mine);
      u.i = want_entry ? 0 : which - base - (of(upto) - u.units);
      u.first = parts + of(pupto) - of(kept);
      return u;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
    parts += __builtin_amdgcn_readlane(pupto, 63);
  }
  return u;
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

template <bool BF16, int NH> struct Shape {
  static constexpr int KROWS = BF16 ? 32 : 16;          // rows of a step
  static constexpr int KT = KROWS / 16;                 // score tiles of a step
  static constexpr int NJ = BF16 ? 4 : 4 * NH;          // 16-byte pieces of a row that a lane holds for the scores
  static constexpr int NV = BF16 ? 8 : 4;               // V rows of a step that a lane holds
  static constexpr int NA = BF16 ? 8 : 4 * NH;          // accumulator tiles
};

// BF16: head width 128.  Float: NH = 1 for widths up to 64, 2 up to 128.  RT: tiles of 16 query rows that a workgroup takes.
// TREE: rows from n_true on are seen as the tree's bits say.
template <bool BF16, int NH, int RT, bool TREE>
__global__ __launch_bounds__(64 * WAVES) void paged_attn_kernel(PagedAttnArgs a, int heads8, int rowblocks) {
  using S = Shape<BF16, NH>;
  constexpr int E = BF16 ? 2 : 4, HDP = BF16 ? 128 : 64 * NH;       // bytes of a value; padded head width
  __shared__ float part_o[WAVES][16][HDP + 4];
  __shared__ float part_m[WAVES][RT * 16], part_l[WAVES][RT * 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
  // row blocks of one unit and head stand eight workgroups apart: on one XCD, whose L2 has the rows after the first
  const int id = blockIdx.x, ug = id / (8 * rowblocks) * 8 + id % 8, rb = id / 8 % rowblocks;
  if (ug >= heads8) return;
  const int head = ug % a.G;
  const Unit u = find_unit(a, ug / a.G, false);
  if (u.b < 0) return;
  const int slot = __builtin_amdgcn_readfirstlane(paged_slot(a.c, a.slots, u.b));
  PagedRows rows = rows_of(a, slot, u.b);
  rows.n = __builtin_amdgcn_readfirstlane(rows.n); rows.nt = __builtin_amdgcn_readfirstlane(rows.nt);
  rows = paged_rows(rows.n, rows.nt, a.window, a.sinks);               // (the wave's, not a lane's)
  const int rep = a.H / a.G, R = a.M * rep;
  const int first = u.i * u.chunk, last = min(first + u.chunk, rows.blocks);
  const int64_t row_bytes = (int64_t)a.G * a.d * E;
  const char* kbase = (const char*)a.c.k + (int64_t)head * a.d * E;
  const char* vbase = (const char*)a.c.v + (int64_t)head * a.d * E;
  const int32_t* table = a.c.table + (int64_t)max(slot, 0) * a.c.W;
  const int in_page = (1 << a.c.shift) - 1;

  // queries: column l16 of tile t is row r of this kv head's R = M * rep rows
  u32x4 q[RT][S::NJ];
  int qm[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = (rb * RT + t) * 16 + l16, m = r / rep;
    qm[t] = m;
    const char* p = (const char*)a.q + ((((int64_t)u.b * a.M + m) * a.H + head * rep + r % rep) * a.d) * E;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const int piece = (4 * j + g4) * 16;
      q[t][j] = r < R && piece < a.d * E ? *(const u32x4*)(p + piece) : u32x4{0, 0, 0, 0};
    }
  }
  f32x4 acc[RT][S::NA];
  float mx[RT], sum[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    mx[t] = -INFINITY; sum[t] = 0.f;
#pragma unroll
    for (int c = 0; c < S::NA; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c2 = fmaxf(a.scale * LOG2E, 1.1754944e-38f);           // (0 * -infinity is no number)

  // ---- the steps of this wave: KROWS rows each, of every WAVES-th block of the unit
  constexpr int SUB = PAGED_BLOCK / S::KROWS;
  const int steps = last > first + wave ? (last - first - wave + WAVES - 1) / WAVES * SUB : 0;
  const int shift = a.c.shift;
  const bool wide = shift >= 4;            // 16 rows of a score tile stand on one page: its number is the wave's, not a lane's
  auto base_of = [&](int s) { return paged_block(rows, first + wave + s / SUB * WAVES) * PAGED_BLOCK + s % SUB * S::KROWS; };
  auto page_of = [&](int row) { return paged_page(table, row, paged_seen(rows, row), shift, a.c.P); };
  // page numbers of a step, a step ahead of the rows: of the tiles, if they stand on one page each
  struct Ahead { int base, whole; int page[S::KT]; };
  auto look = [&](int s) BEAGLE_INLINE_LAMBDA {
    Ahead h;
    h.base = __builtin_amdgcn_readfirstlane(s < steps ? base_of(s) : rows.n);
    h.whole = wide && paged_all_seen(rows, h.base, S::KROWS);
#pragma unroll
    for (int t = 0; t < S::KT; ++t) h.page[t] = h.whole ? table[(h.base + 16 * t) >> shift] : 0;
    return h;
  };
  // (an unreadable page number: the step goes row by row)
  auto settle = [&](Ahead& h) BEAGLE_INLINE_LAMBDA {
#pragma unroll
    for (int t = 0; t < S::KT; ++t) {
      h.page[t] = __builtin_amdgcn_readfirstlane(h.page[t]);
      if ((unsigned)h.page[t] >= (unsigned)a.c.P) h.whole = 0;
    }
  };
  uint32_t koff[S::NJ], voff[4][NH];       // of a lane's pieces, from the first row of a tile
#pragma unroll
  for (int j = 0; j < S::NJ; ++j) koff[j] = (uint32_t)(l16 * row_bytes) + (4 * j + g4) * 16;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int h = 0; h < NH; ++h) voff[i][h] = (uint32_t)((4 * g4 + i) * row_bytes) + (16 * h + l16) * 16;
  u32x4 k[S::KT][S::NJ], v[S::NV][NH];
  // K rows, one in each lane's l16
  auto request_k = [&](const Ahead& h) BEAGLE_INLINE_LAMBDA {
#pragma unroll
    for (int t = 0; t < S::KT; ++t) {
      if (h.whole) {
        const char* src = kbase + (((int64_t)h.page[t] << shift) + ((h.base + 16 * t) & in_page)) * row_bytes;
#pragma unroll
        for (int j = 0; j < S::NJ; ++j)
          k[t][j] = BF16 || (4 * j + g4) * 16 < a.d * E ? *(const u32x4*)(src + koff[j]) : u32x4{0, 0, 0, 0};
      } else {
        const int row = h.base + 16 * t + l16, p = page_of(row);
        const char* src = p >= 0 ? kbase + (((int64_t)p << shift) + (row & in_page)) * row_bytes : (const char*)zero_row;
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) {
          const int piece = (4 * j + g4) * 16;
          k[t][j] = *(const u32x4*)(BF16 || piece < a.d * E ? src + piece : (const char*)zero_row);
        }
      }
    }
  };
  // V rows, four neighbours in each lane's g4 (one page: its rows are a multiple of four)
  auto request_v = [&](const Ahead& h) BEAGLE_INLINE_LAMBDA {
#pragma unroll
    for (int t = 0; t < S::KT; ++t) {
      if (h.whole) {
        const char* src = vbase + (((int64_t)h.page[t] << shift) + ((h.base + 16 * t) & in_page)) * row_bytes;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int n = 0; n < NH; ++n)
            v[4 * t + i][n] = BF16 || (16 * n + l16) * 16 < a.d * E ? *(const u32x4*)(src + voff[i][n]) : u32x4{0, 0, 0, 0};
      } else {
        const int r0 = h.base + 16 * t + 4 * g4, p = paged_page(table, r0, r0 < rows.n, shift, a.c.P);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool seen = p >= 0 && paged_seen(rows, r0 + i);
          const char* src = seen ? vbase + (((int64_t)p << shift) + ((r0 + i) & in_page)) * row_bytes : (const char*)zero_row;
#pragma unroll
          for (int n = 0; n < NH; ++n) {
            const int piece = (16 * n + l16) * 16;
            v[4 * t + i][n] = *(const u32x4*)(BF16 || piece < a.d * E ? src + piece : (const char*)zero_row);
          }
        }
      }
    }
  };
  Ahead now = look(0), next = look(1);
  settle(now);
  if (steps > 0) { request_k(now); request_v(now); }
  for (int s = 0; s < steps; ++s) {
    // ---- scores
    f32x4 sc[RT][S::KT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int kt = 0; kt < S::KT; ++kt) {
        sc[t][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) {
          if constexpr (BF16) sc[t][kt] = mfma_bf16(k[kt][j], q[t][j], sc[t][kt]);
          else
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[t][kt] = mfma_f32(__uint_as_float(k[kt][j][e]), __uint_as_float(q[t][j][e]), sc[t][kt]);
        }
      }
    // the registers of K are free: the next step's rows travel while this one's probabilities are computed
    settle(next);
    if (s + 1 < steps) request_k(next);
    const Ahead after = look(s + 2);
    bool seen[S::KT][4];
    if (!now.whole) {
#pragma unroll
      for (int kt = 0; kt < S::KT; ++kt) {
        const int r0 = now.base + 16 * kt + 4 * g4;
        const bool there = paged_page(table, r0, r0 < rows.n, shift, a.c.P) >= 0;      // (a page number that is none hides its rows)
#pragma unroll
        for (int i = 0; i < 4; ++i) seen[kt][i] = there && paged_seen(rows, r0 + i);
      }
    }
    // A drafted row that only some queries see may hold what is no number, which the others must not meet (0 * NaN is
    // NaN).  The matrix instructions mix all rows into all queries, so such a step adds row by row where it is seen.
    [[maybe_unused]] bool odd = false;
    if constexpr (TREE)
      if (now.base + S::KROWS > rows.nt) {
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
        odd = __ballot(top == 0x7f800000u) != 0;
      }
    // ---- running maximum and sum, probabilities
    float p[RT][S::KT][4];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (!now.whole) {
#pragma unroll
        for (int kt = 0; kt < S::KT; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            bool see = seen[kt][i];
            if constexpr (TREE) {
              const int bit = now.base + 16 * kt + 4 * g4 + i - rows.nt;
              if (see && bit >= 0)
                see = qm[t] < a.M && (bit >> 5) < a.words &&
                      (a.tree[((int64_t)u.b * a.M + qm[t]) * a.words + (bit >> 5)] >> (bit & 31) & 1u);
            }
            if (!see) sc[t][kt][i] = -INFINITY;
          }
      }
      float top = sc[t][0][0];
#pragma unroll
      for (int e = 1; e < 4 * S::KT; ++e) top = fmaxf(top, sc[t][e / 4][e % 4]);
      const float most = fmaxf(mx[t], max_over_keys(top) * c2), safe = most == -INFINITY ? 0.f : most;
      if (__any(most > mx[t])) {
        const float shrink = exp2_fast(mx[t] - safe);
        sum[t] *= shrink;
#pragma unroll
        for (int c = 0; c < S::NA; ++c) acc[t][c] *= shrink;
        mx[t] = most;
      }
#pragma unroll
      for (int kt = 0; kt < S::KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) { p[t][kt][i] = exp2_fast(fmaf(sc[t][kt][i], c2, -safe)); sum[t] += p[t][kt][i]; }
    }
    // ---- O^T += V^T P^T
    if (TREE && odd) {
      float* mine = part_o[wave][l16];       // (free until the end)
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int kt = 0; kt < S::KT; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i) mine[16 * kt + 4 * g4 + i] = sc[t][kt][i] == -INFINITY ? -1.f : p[t][kt][i];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (int j = 0; j < S::KROWS; ++j) {
          const float w = mine[j];
          const int row = now.base + j, pg = page_of(row);
          if (w == -1.f || pg < 0) continue;
          const char* src = vbase + (((int64_t)pg << shift) + (row & in_page)) * row_bytes;
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
    } else if constexpr (BF16) {
      // a probability as two bf16 numbers, 16 bits in all: the matrix pipe has the time, and the rounding of one
      // would cost the output as much again as its own (2^-9)
      u32x4 hi[RT], lo[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = p[t][i >> 1][2 * (i & 1)], y = p[t][i >> 1][2 * (i & 1) + 1];
          hi[t][i] = pack_bf16x2(x, y);
          lo[t][i] = pack_bf16x2(x - __uint_as_float(hi[t][i] << 16), y - __uint_as_float(hi[t][i] & 0xffff0000u));
        }
#pragma unroll
      for (int c = 0; c < 8; ++c) {       // channels 8 l16 + c
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = __builtin_amdgcn_perm(v[2 * i + 1][0][c >> 1], v[2 * i][0][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          acc[t][c] = mfma_bf16(w, hi[t], acc[t][c]);
          acc[t][c] = mfma_bf16(w, lo[t], acc[t][c]);
        }
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
    if (s + 1 < steps) request_v(next);
    now = next;
    next = after;
  }

  // ---- the waves' shares, then the unit's result
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float l = sum[t];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g4 == 0) { part_m[wave][16 * t + l16] = mx[t]; part_l[wave][16 * t + l16] = l; }
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
        *(f32x4*)&part_o[wave][l16][ch] = f32x4{acc[t][c][i], acc[t][c + 1][i], acc[t][c + 2][i], acc[t][c + 3][i]};
      }
    __syncthreads();
    const int col = threadIdx.x >> 4, r = (rb * RT + t) * 16 + col;
    if (r >= R) continue;
    float m = -INFINITY, l = 0.f, w[WAVES];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) m = fmaxf(m, part_m[i][16 * t + col]);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      w[i] = m == -INFINITY ? 0.f : exp2_fast(part_m[i][16 * t + col] - m);
      l += part_l[i][16 * t + col] * w[i];
    }
    const int qi = r / rep, h = head * rep + r % rep;
    const bool whole = u.units == 1;
    const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
    const int64_t prow = ((int64_t)(u.first + u.i) * a.G + head) * R + r;      // (whole: not used)
#pragma unroll
    for (int half = 0; half < HDP / 64; ++half) {
      const int ch = 64 * half + 4 * (threadIdx.x & 15);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < WAVES; ++i) o += *(const f32x4*)&part_o[i][col][ch] * w[i];
      o *= inv;
      if (!whole) { *(f32x4*)(a.part + prow * HDP + ch) = o; continue; }
      if (ch >= a.d) continue;
      const int64_t at = (((int64_t)u.b * a.M + qi) * a.H + h) * a.d + ch;
      if constexpr (BF16) *(uint2*)((bf16_t*)a.o + at) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
      else *(f32x4*)((float*)a.o + at) = o;
    }
    if ((threadIdx.x & 15) == 0) {
      if (whole) a.lse[((int64_t)u.b * a.H + h) * a.M + qi] = (m + __log2f(l)) * LN2;
      else *(float2*)(a.ml + prow * 2) = make_float2(m, l);
    }
  }
}

// The units of an entry, in order: eight of them at a time (a group of 32 lanes each), then the groups through LDS.
template <bool BF16, int HDP>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int GROUPS = 256 / (HDP / 4);
  __shared__ float so[GROUPS][HDP];
  __shared__ float sm[GROUPS], sl[GROUPS];
  const int rep = a.H / a.G, R = a.M * rep;
  const Unit u = find_unit(a, blockIdx.y, true);
  if (u.units <= 1) return;
  const int h = blockIdx.x % a.H, qi = blockIdx.x / a.H, head = h / rep, r = qi * rep + h % rep;
  const int group = threadIdx.x / (HDP / 4), ch = 4 * (threadIdx.x % (HDP / 4));
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  for (int i = group; i < u.units; i += GROUPS) {
    const int64_t prow = ((int64_t)(u.first + i) * a.G + head) * R + r;
    const float2 ml = *(const float2*)(a.ml + prow * 2);
    const f32x4 po = *(const f32x4*)(a.part + prow * HDP + ch);
    const float now = fmaxf(m, ml.x), safe = now == -INFINITY ? 0.f : now;
    const float w0 = exp2_fast(m - safe), w1 = exp2_fast(ml.x - safe);
    o = o * w0 + po * w1;
    l = l * w0 + ml.y * w1;
    m = now;
  }
  *(f32x4*)&so[group][ch] = o;
  if (ch == 0) { sm[group] = m; sl[group] = l; }
  __syncthreads();
  if (group) return;
  for (int i = 1; i < GROUPS; ++i) {
    const float now = fmaxf(m, sm[i]), safe = now == -INFINITY ? 0.f : now;
    const float w0 = exp2_fast(m - safe), w1 = exp2_fast(sm[i] - safe);
    o = o * w0 + *(const f32x4*)&so[i][ch] * w1;
    l = l * w0 + sl[i] * w1;
    m = now;
  }
  if (ch == 0) a.lse[((int64_t)u.b * a.H + h) * a.M + qi] = (m + __log2f(l)) * LN2;
  if (ch >= a.d) return;
  o *= l == 0.f ? 0.f : 1.f / l;
  const int64_t at = (((int64_t)u.b * a.M + qi) * a.H + h) * a.d + ch;
  if constexpr (BF16) *(uint2*)((bf16_t*)a.o + at) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
  else *(f32x4*)((float*)a.o + at) = o;
}

constexpr int AIM = 1024;                  // workgroups
constexpr int MAX_TILES = 4;               // of 16 query rows that a workgroup takes
struct Tiles { int each, blocks; };        // tiles of a workgroup, workgroups that the rows of a kv head take
Tiles tiles_of(int R) {
  const int all = (R + 15) / 16, blocks = (all + MAX_TILES - 1) / MAX_TILES;
  return {(all + blocks - 1) / blocks, blocks};
}
int units_aimed(int R, int G) {
  const int64_t per = (int64_t)G * tiles_of(R).blocks;
  return per < AIM ? (int)(AIM / per) : 1;
}

}  // namespace

// Partial sums: only entries of several units have them, and those are at most twice the units aimed at.
size_t paged_attn_ws_bytes(int32_t M, int32_t H, int32_t G) {
  const int64_t R = (int64_t)M * (H / G);
  return (size_t)2 * units_aimed((int)R, G) * G * R * (128 + 2) * sizeof(float);
}

void launch_paged_attn(bool bf16, PagedAttnArgs a, void* ws, hipStream_t s) {
  const int R = a.M * (a.H / a.G);
  const Tiles tiles = tiles_of(R);
  a.target = units_aimed(R, a.G);
  a.least = WAVES;
  const int64_t rows = (int64_t)2 * a.target * a.G * R;
  a.part = (float*)ws;
  a.ml = a.part + rows * 128;
  const int heads8 = (a.target + a.B) * a.G;
  const dim3 grid((unsigned)((heads8 + 7) / 8 * 8 * tiles.blocks)), wg(64 * WAVES);
  const bool tree = a.n_true != nullptr, narrow = !bf16 && a.d <= 64;
  {
    ProfScope ps("paged_attn", s);
    auto go = [&](auto bf_, auto nh_, auto rt_) {
      constexpr bool BF = decltype(bf_)::value != 0;
      constexpr int NH = decltype(nh_)::value, RT = decltype(rt_)::value;
      if (tree) hipLaunchKernelGGL((paged_attn_kernel<BF, NH, RT, true>), grid, wg, 0, s, a, heads8, tiles.blocks);
      else hipLaunchKernelGGL((paged_attn_kernel<BF, NH, RT, false>), grid, wg, 0, s, a, heads8, tiles.blocks);
    };
    auto with = [&](auto bf_, auto nh_) {
      if (tiles.each == 1) go(bf_, nh_, int_c<1>{});
      else if (tiles.each == 2) go(bf_, nh_, int_c<2>{});
      else if (tiles.each == 3) go(bf_, nh_, int_c<3>{});
      else go(bf_, nh_, int_c<4>{});
    };
    if (bf16) with(int_c<1>{}, int_c<1>{});
    else if (narrow) with(int_c<0>{}, int_c<1>{});
    else with(int_c<0>{}, int_c<2>{});
  }
  // no entry can have two units: nothing to join
  if ((a.bound + PAGED_BLOCK - 1) / PAGED_BLOCK <= a.least) return;
  ProfScope ps("paged_join", s);
  const dim3 jg((unsigned)(a.H * a.M), (unsigned)a.B);
  if (bf16) hipLaunchKernelGGL((paged_join_kernel<true, 128>), jg, dim3(256), 0, s, a);
  else if (narrow) hipLaunchKernelGGL((paged_join_kernel<false, 64>), jg, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_join_kernel<false, 128>), jg, dim3(256), 0, s, a);
}

}  // namespace beagle
