// Attention to a few pages of a long context: bounds of every page's keys, the pages that they put first, attention over those.
//
//   lo_pc = min_j k_jc, hi_pc = max_j k_jc over the rows j of page p;   score_p = max_r sum_c max(q_rc lo_pc, q_rc hi_pc),
//
// which no <q_r, k_j> of the page exceeds.  An entry's first pages and its last ones are always seen; of those between them a kv
// head sees the n_select with the highest scores.
#include "paged_attend.h"
#include "attn_tiles.h"
#include "paged_pick.h"

namespace beagle {
namespace {

// ------------------------------------------------------------------ bounds
// One workgroup for a page and 64 pieces of 16 bytes of its rows; the waves take the rows in turns, eight requests of a lane on their way, and join through
// LDS.  Bound: the keys' bytes.  6 sequences of up to 8000 rows of 32 heads (bf16, pages of 64, 248 MB of keys) 49 us, 5.2 TB/s (MI355X); 64 sequences of 5
// new rows each 6.3: one launch and three dependent trips.
template <bool BF16>
__global__ __launch_bounds__(256) void paged_bounds_kernel(PagedCache c, int G, int d, int bound, const int32_t* slots, const int32_t* first,
                                                           char* bounds) {
  constexpr int E = BF16 ? 2 : 4, N = 16 / E;
  __shared__ float part[4][64][2 * N + 1];
  const int b = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int slot = paged_slot(c, slots, b);
  const int n = min(paged_len(c, slot), bound);
  const int from = (first ? max(first[b], 0) : 0) >> c.shift, to = n >> c.shift;
  const int pieces = G * d / N, groups = (pieces + 63) / 64;
  const int64_t row_bytes = (int64_t)G * d * E;
  const int64_t units = (int64_t)max(to - from, 0) * groups;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int page = c.table[(int64_t)slot * c.W + from + (int)(u / groups)], piece = (int)(u % groups) * 64 + lane;
    if ((unsigned)page >= (unsigned)c.P) continue;           // (the same in all lanes)
    float lo[N], hi[N];
#pragma unroll
    for (int i = 0; i < N; ++i) { lo[i] = INFINITY; hi[i] = -INFINITY; }
    const addr_t src = (addr_t)c.k + ((int64_t)page << c.shift) * row_bytes + 16 * min(piece, pieces - 1);
#pragma unroll 8
    for (int j = wave; j < 1 << c.shift; j += 4) {
      const u32x4 x = load16(src + j * row_bytes);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float v = BF16 ? __uint_as_float(i & 1 ? x[i / 2] & 0xffff0000u : x[i / 2] << 16) : __uint_as_float(x[i % 4]);
        lo[i] = fminf(lo[i], v); hi[i] = fmaxf(hi[i], v);
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) { part[wave][lane][i] = lo[i]; part[wave][lane][N + i] = hi[i]; }
    __syncthreads();
    if (wave < 2 && piece < pieces) {                        // wave 0: the least, wave 1: the greatest
      float v[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float p0 = part[0][lane][wave * N + i], p1 = part[1][lane][wave * N + i], p2 = part[2][lane][wave * N + i], p3 = part[3][lane][wave * N + i];
        v[i] = wave ? fmaxf(fmaxf(p0, p1), fmaxf(p2, p3)) : fminf(fminf(p0, p1), fminf(p2, p3));
      }
      const int head = piece * N / d, ch = piece * N % d;
      char* dst = bounds + ((((int64_t)page * G + head) * 2 + wave) * d + ch) * E;
      if constexpr (BF16) *(u32x4*)dst = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
      else *(f32x4*)dst = f32x4{v[0], v[1], v[2], v[3]};
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ selection
// The order of the pages is that of sums in 64 bits, rounded to float; but those are needed only where a page's place is in doubt.  The scores
// are first taken from matrix instructions, sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c, and are then off by at most E:
//   64 additions of a piece's products, each off by at most 2^-23 of the magnitudes |q_c x_c| of the piece, and 4 of pieces, by 2^-24 of all,
//   less than 1.0625 * 2^-17 of sum_c |q_c x_c| <= |q| |(lo, hi)| together; inputs and sums below 2^-126 may count as zero.
// (The norms are summed from squares, of which those below 2^-126 may count as zero too, together a norm of less than 2^-58.)
// With t the n_select-th largest of them, the true one is within E of t: a page above t + 2 E is picked, one below t - 2 E is not, and of those
// between (most often only the one that t comes from) the true scores are taken where they are more than are still to be picked.
// Infinities and what is no number make E infinite, and all scores true ones.
//
// Bound: the bounds' bytes, and of little work the chain of a launch, lengths, page numbers, bounds, and the picking (some 4 us).  Measured (MI355X, bf16, a graph's
// replays): 160 heads of up to 1008 pages, 10 queries (61 MB) 22 us, 256 heads of up to 304 pages, 4 queries (23 MB) 13, 32 heads of 179 pages 9.5.  With
// all scores in 64 bits the first took 120 us, the second 102: the vector pipe's double rate.
constexpr int SELECT_HELD = 8192;          // scores that a workgroup holds

struct Span { int lead, count; const int32_t* table; };
// the pages that an entry's selection is made of: `count` of them from `lead` on
__device__ __forceinline__ Span span_of(const PagedSelectArgs& a, int b) {
  const int slot = paged_slot(a.c, a.slots, b);
  const int n = min(paged_len(a.c, slot), a.bound);
  const PagedPick p = paged_pick(n, a.n_true ? a.n_true[b] : INT32_MAX, a.window, a.sinks, a.n_select, a.c.shift);
  return {p.lead, p.listed + p.gap, a.c.table + (int64_t)max(slot, 0) * a.c.W};
}

// Sixteen pages' bounds of each wave on their way (bf16): sixteen lanes ask for a whole row of 256 bytes.  (Asked for in the order that the matrix instructions
// take, 64 bytes of each of sixteen rows at a time, 96 heads of 1992 pages took 39 us, not 28.)  Chunk c of row r is at c ^ swz(r).
struct Staged { u32x4 x[2][SELECT_WAVES][2][16 * 16]; };

template <bool BF16> struct Rows {         // sixteen rows as the matrix instructions take them: lane % 16 is the row, lane / 16 the piece of 16 bytes
  static constexpr int E = BF16 ? 2 : 4, NJ = BF16 ? 4 : 8;
  u32x4 x[NJ];
  __device__ __forceinline__ void load(addr_t row, int d, bool there) {
    const int g4 = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int j = 0; j < NJ; ++j) x[j] = load16(there && (BF16 || (4 * j + g4) * 16 < d * E) ? row + (4 * j + g4) * 16 : (addr_t)zero_row);
  }
  // the positive, or the negative, values; the others as zero
  __device__ __forceinline__ Rows part(bool negative) const {
    Rows r;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t v = x[j][i];          // (a bit cast of the element itself takes the first one's bits)
        uint32_t sign;
        if constexpr (BF16) {
          typedef short i16x2 __attribute__((ext_vector_type(2)));
          sign = __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, v) >> 15);
        } else {
          sign = (uint32_t)((int)v >> 31);
        }
        r.x[j][i] = v & (negative ? sign : ~sign);
      }
    return r;
  }
  // the sum of their squares
  __device__ __forceinline__ float squares() const {
    float s[4] = {};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t v = x[j][i];
        if constexpr (BF16) {
          typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
          s[i] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, v), __builtin_bit_cast(bf16x2, v), s[i], false);
        } else {
          s[i] = fmaf(__uint_as_float(v), __uint_as_float(v), s[i]);
        }
      }
    return (s[0] + s[1]) + (s[2] + s[3]);
  }
};
// Register e: query row 4 (lane / 16) + e of sixteen, page lane % 16.  (Pieces of 32 channels, floats of 16, add up by themselves: less rounding, and
// few instructions wait for another's sum.)
template <bool BF16> __device__ __forceinline__ f32x4 product(const Rows<BF16>& minus, const Rows<BF16>& plus, const Rows<BF16>& lo, const Rows<BF16>& hi) {
  constexpr int NJ = Rows<BF16>::NJ;
  f32x4 s[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](const Rows<BF16>& q, const Rows<BF16>& x) BEAGLE_INLINE_LAMBDA {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if constexpr (BF16) s[j] = mfma_bf16(q.x[j], x.x[j], s[j]);
      else
#pragma unroll
        for (int e = 0; e < 4; ++e) s[j] = mfma_f32(__uint_as_float(q.x[j][e]), __uint_as_float(x.x[j][e]), s[j]);
  };
  add(minus, lo);
  add(plus, hi);
#pragma unroll
  for (int n = NJ / 2; n > 0; n /= 2)
#pragma unroll
    for (int j = 0; j < n; ++j) s[j] += s[j + n];
  return s[0];
}
// Scores of pages [from, to) of the span by matrix instructions, sixteen at a time to each wave.  Returns the wave's share of their extent.
// (Loops that are not unrolled: all of this runs once or a few times, and instructions that come from memory take longer than they run.)
template <bool BF16>
__device__ __forceinline__ Extent score_pages(const PagedSelectArgs& a, Staged* staged, const int32_t* table, int b, int g, int from, int to, uint32_t* out) {
  constexpr int E = BF16 ? 2 : 4, STEP = SELECT_WAVES * 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
  const int rep = a.H / a.G, R = a.M * rep;
  auto query = [&](int first) {
    const int r = first + l16;
    Rows<BF16> q;
    q.load((addr_t)a.q + (((int64_t)b * a.M + r / rep) * a.H + g * rep + r % rep) * a.d * E, a.d, r < R);
    return q;
  };
  const int first = from + wave * 16;
  // a lane's number of the wave's next four turns: lane % 16 of turn lane / 16 (behind the end the last page again)
  auto numbers_of = [&](int i0) { return table[min(i0 + g4 * STEP + l16, to - 1)]; };
  int numbers = first < to ? numbers_of(first) : -1;
  Rows<BF16> q = query(0), plus = q.part(false), minus = q.part(true);
  // What is loaded into registers is waited for here, and where it is loaded: later the wait would be one for requests into LDS, too, that the
  // compiler does not count.
  if constexpr (BF16) {
    asm volatile("" : "+v"(numbers));
#pragma unroll
    for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(q.x[j]), "+v"(plus.x[j]), "+v"(minus.x[j]));
  }
  uint32_t of_pages = 0, of_queries = 0;                     // the largest sums of squares, as bits; what is no number is above all
  Extent x = {0.f, INFINITY, -INFINITY};
  struct Pages { Rows<BF16> lo, hi; bool there; };
  auto there = [&](int number) { return (unsigned)number < (unsigned)a.c.P; };
  const int64_t row_bytes = (int64_t)2 * a.d * E;
  auto request = [&](int turn, int stage) BEAGLE_INLINE_LAMBDA {                  // (bf16)
    const uint32_t lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uintptr_t)(tiles::lds_void_ptr)staged->x[stage][wave][0]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int number = __shfl(numbers, 16 * (turn & 3) + 4 * j + g4);
      const addr_t at = (there(number) ? (addr_t)a.bounds + ((int64_t)number * a.G + g) * row_bytes : (addr_t)zero_row) + 16 * (l16 ^ tiles::swz(4 * j + g4));
      load_to_lds(at, lds + 1024 * j);
      load_to_lds(at + 256, lds + 4096 + 1024 * j);
    }
  };
  auto take = [&](Pages& p, int page, int stage) BEAGLE_INLINE_LAMBDA {
    p.there = there(page);
    if constexpr (BF16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = 16 * l16 + ((4 * j + g4) ^ tiles::swz(l16));
        p.lo.x[j] = staged->x[stage][wave][0][at];
        p.hi.x[j] = staged->x[stage][wave][1][at];
      }
    } else {
      const addr_t at = (addr_t)a.bounds + ((int64_t)page * a.G + g) * row_bytes;
      p.lo.load(at, a.d, p.there);
      p.hi.load(at + a.d * E, a.d, p.there);
    }
  };
  auto score = [&](const Pages& p, int i0) BEAGLE_INLINE_LAMBDA {
    float best = -INFINITY;
#pragma unroll 1
    for (int t = 0; t < R; t += 16) {
      if (R > 16) { q = query(t); plus = q.part(false); minus = q.part(true); }
      if (i0 == first) of_queries = max(of_queries, __float_as_uint(q.squares()) & 0x7fffffffu);   // (while the bounds are on their way)
      const f32x4 s = product(minus, plus, p.lo, p.hi);
#pragma unroll
      for (int e = 0; e < 4; ++e) best = fmaxf(best, t + 4 * g4 + e < R ? s[e] : -INFINITY);
    }
    of_pages = max(of_pages, __float_as_uint(p.lo.squares() + p.hi.squares()) & 0x7fffffffu);
    best = as_float(over_rows(__float_as_uint(best), MaxOf()));
    const float v = p.there ? best : -INFINITY;
    if (g4 == 0 && i0 + l16 < to) out[i0 + l16] = __float_as_uint(v);
    x.most = fmaxf(x.most, v);
    x.least = fminf(x.least, v == -INFINITY ? INFINITY : v);
  };
  // (the next sixteen pages travel meanwhile; of floats there is no room for them)
  if (BF16 && first < to) request(0, 0);
  int turn = 0;
#pragma unroll 1
  for (int i0 = first; i0 < to; i0 += STEP, ++turn) {
    Pages p;
    const int page = __shfl(numbers, 16 * (turn & 3) + l16);
    if ((turn & 3) == 3) {
      numbers = numbers_of(i0 + STEP);
      if (BF16) asm volatile("" : "+v"(numbers));
    }
    if constexpr (BF16) {
      if (i0 + STEP < to) {
        request(turn + 1, (turn + 1) & 1);
        tiles::wait_vmem_n<8>();
      } else {
        tiles::wait_vmem();
      }
      asm volatile("" ::: "memory");       // (nothing of LDS is read before)
    }
    take(p, page, turn & 1);
    score(p, i0);
  }
  // (a row's lanes have their largest parts of all tiles: together no less than any query's, or page's)
  auto norm = [&](uint32_t squares) { return sqrtf(as_float(over_row(over_rows(squares, SumOf()), MaxBits()))); };
  const float nq = norm(of_queries), nx = norm(of_pages), size = nq * nx;        // (finite: and so is every sum on the way)
  x.off = 1.01f * 0x1.1p-17f * (size + 0x1p-58f * (nq + nx) + 0x1p-100f);
  if (!(size < INFINITY && x.off < INFINITY)) x.off = INFINITY;
  x.least = as_float(over_all(__float_as_uint(x.least), MinOf()));
  x.most = as_float(over_all(__float_as_uint(x.most), MaxOf()));
  return x;
}

// <q_r, the bounds> for page i of the span and one query row in 64 bits, by sixteen lanes; -infinity where there is no such page
template <bool BF16>
__device__ __forceinline__ float true_score(const PagedSelectArgs& a, const int32_t* table, int b, int g, int i, int r) {
  constexpr int E = BF16 ? 2 : 4;
  const int lane = threadIdx.x & 15, rep = a.H / a.G;
  const int page = table[i];
  const bool there = (unsigned)page < (unsigned)a.c.P;
  const addr_t at_q = (addr_t)a.q + (((int64_t)b * a.M + r / rep) * a.H + g * rep + r % rep) * a.d * E;
  const addr_t at_lo = (addr_t)a.bounds + ((int64_t)(there ? page : 0) * a.G + g) * 2 * a.d * E, at_hi = at_lo + a.d * E;
  double s = 0.0;
#pragma unroll
  for (int h = 0; h < (BF16 ? 1 : 2); ++h) {                 // channels 8 lane .., floats 4 lane + 64 h ..
    const int byte = 16 * lane + 256 * h;
    const bool in = byte < a.d * E;
    const u32x4 q = load16(in ? at_q + byte : (addr_t)zero_row), lo = load16(in ? at_lo + byte : (addr_t)zero_row),
                hi = load16(in ? at_hi + byte : (addr_t)zero_row);
#pragma unroll
    for (int e = 0; e < 16 / E; ++e) {
      auto value = [&](const u32x4& x) { return BF16 ? as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16) : as_float(x[e % 4]); };
      const float v = value(q);
      if (v > 0.f) s = fma((double)v, (double)value(hi), s);
      else if (v < 0.f) s = fma((double)v, (double)value(lo), s);
    }
  }
#pragma unroll
  for (int k = 1; k < 16; k *= 2) s += __shfl_xor(s, k);
  return there ? (float)s : -INFINITY;
}

// An entry's and head's pages from their scores (pick_pages)
template <bool BF16, bool MEMORY>
__device__ __forceinline__ void pick(const PagedSelectArgs& a, PickShared& sh, const Span& span, int b, int g, uint32_t* scores, const Extent& x, int32_t* out) {
  const int32_t* table = span.table + span.lead;
  pick_pages<MEMORY>(sh, span.count, a.n_select, span.lead, a.M * (a.H / a.G), scores, x, out,
                     [&](int i, int r) BEAGLE_INLINE_LAMBDA { return true_score<BF16>(a, table, b, g, i, r); });
}

// every page is picked
__device__ __forceinline__ bool picks_all(const PagedSelectArgs& a, const Span& span, int32_t* out) {
  if (span.count > a.n_select) return false;
  for (int i = threadIdx.x; i < a.n_select; i += SELECT_THREADS) out[i] = i < span.count ? span.lead + i : -1;
  return true;
}

// One workgroup for an entry and head: scores in LDS, and the pages from them.
template <bool BF16>
__global__ __launch_bounds__(SELECT_THREADS) void paged_select_kernel(PagedSelectArgs a) {
  __shared__ union { PickShared pick; Staged staged[BF16 ? 1 : 0]; } sh;
  __shared__ uint32_t scores[SELECT_HELD];
  // Workgroups go round the chip's eight dies.  Heads g, g + 8, .. of one entry on one die would ask for addresses that are alike in their
  // lowest 4 KB, two of the sixteen channels of the die's cache; so each has its heads one behind the other.
  const uint32_t all = (uint32_t)a.B * a.G, each = (all + 7) / 8;
  for (uint32_t i = blockIdx.x; i < 8 * each; i += gridDim.x) {
    const uint32_t bg = i % 8 * each + i / 8;
    if (bg >= all) continue;
    const int b = (int)(bg / (uint32_t)a.G), g = (int)(bg % (uint32_t)a.G);
    const Span span = span_of(a, b);
    int32_t* out = a.pages + (int64_t)bg * a.n_select;
    if (picks_all(a, span, out)) continue;
    const Extent x = score_pages<BF16>(a, sh.staged, span.table + span.lead, b, g, 0, span.count, scores);
    if (BF16) __syncthreads();
    pick<BF16, false>(a, sh.pick, span, b, g, scores, x, out);
  }
}

// Few entries and heads of many pages: scores by as many workgroups as fill the chip, in memory, then the pages.
constexpr int SELECT_CHUNK = 16 * SELECT_WAVES;
template <bool BF16>
__global__ __launch_bounds__(SELECT_THREADS) void paged_score_kernel(PagedSelectArgs a, int chunks) {
  __shared__ u32x4 staged[BF16 ? sizeof(Staged) / 32 : 1];   // (the first half: no wave has a second turn)
  const int b = blockIdx.z;
  const Span span = span_of(a, b);
  for (int g = blockIdx.y; g < a.G; g += gridDim.y)
    for (int chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
      const int64_t bg = (int64_t)b * a.G + g;
      const int from = chunk * SELECT_CHUNK, to = min(from + SELECT_CHUNK, span.count);
      Extent x = {0.f, INFINITY, -INFINITY};
      if (span.count > a.n_select && from < to) x = score_pages<BF16>(a, (Staged*)staged, span.table + span.lead, b, g, from, to, a.scores + bg * a.width);
      if ((threadIdx.x & 63) == 0) ((Extent*)a.extents)[(bg * chunks + chunk) * SELECT_WAVES + (threadIdx.x >> 6)] = x;
    }
}
template <bool BF16>
__global__ __launch_bounds__(SELECT_THREADS) void paged_pick_kernel(PagedSelectArgs a, int chunks) {
  __shared__ PickShared sh;
  __shared__ uint32_t held[SELECT_HELD];
  const int b = blockIdx.y;
  const Span span = span_of(a, b);
  for (int g = blockIdx.x; g < a.G; g += gridDim.x) {
    const int64_t bg = (int64_t)b * a.G + g;
    int32_t* out = a.pages + bg * a.n_select;
    if (picks_all(a, span, out)) continue;
    Extent x = {0.f, INFINITY, -INFINITY};
    for (int i = threadIdx.x; i < chunks * SELECT_WAVES; i += SELECT_THREADS) {
      const Extent y = ((const Extent*)a.extents)[bg * chunks * SELECT_WAVES + i];
      x = Extent{fmaxf(x.off, y.off), fminf(x.least, y.least), fmaxf(x.most, y.most)};
    }
    x.off = as_float(over_all(__float_as_uint(x.off), MaxBits()));
    x.least = as_float(over_all(__float_as_uint(x.least), MinOf()));
    x.most = as_float(over_all(__float_as_uint(x.most), MaxOf()));
    uint32_t* scores = a.scores + bg * a.width;
    if (span.count > SELECT_HELD) {
      pick<BF16, true>(a, sh, span, b, g, scores, x, out);
      continue;
    }
    for (int i = threadIdx.x; i < span.count; i += SELECT_THREADS) held[i] = scores[i];
    pick<BF16, false>(a, sh, span, b, g, held, x, out);
  }
}

}  // namespace

// The attention over listed pages is that over all rows (paged_attn.hip) with the visible rows counted through the list, its page numbers held in LDS.
// Bound: HBM, in pieces of a head's 256 bytes of a row.  Measured (MI355X, bf16, a graph's replays): 32 entries of 4 queries, 32 / 8 heads, 40 pages of 64 rows
// and 516 rows or more (414 MB) 92 us, 4.5 TB/s; 4 entries of 10 queries under a tree, 40 heads, 100 pages of 32 and 566 rows or more (313 MB) 71 us, 4.4 TB/s.
void launch_paged_blocks(bool bf16, PagedAttnArgs a, void* ws, hipStream_t s) { launch_attend<LISTED>(bf16, a, ws, s); }

void launch_paged_bounds(bool bf16, const PagedCache& c, int32_t B, int32_t G, int32_t d, int32_t bound, const int32_t* slots,
                         const int32_t* first, void* bounds, hipStream_t s) {
  ProfScope ps("paged_bounds", s);
  const int64_t pages = bound >> c.shift, groups = ((int64_t)G * d / (bf16 ? 8 : 4) + 63) / 64;
  if (pages < 1) return;                                     // (no page can be whole)
  const int64_t units = pages * groups, each = (4096 + B - 1) / B;
  const dim3 grid((unsigned)(units < each ? units : each), (unsigned)B);
  if (bf16) hipLaunchKernelGGL((paged_bounds_kernel<true>), grid, dim3(256), 0, s, c, G, d, bound, slots, first, (char*)bounds);
  else hipLaunchKernelGGL((paged_bounds_kernel<false>), grid, dim3(256), 0, s, c, G, d, bound, slots, first, (char*)bounds);
}

static int32_t select_width(const PagedCache& c, int32_t bound) {
  const int32_t pages = bound >> c.shift;
  return pages < 1 ? 1 : pages < c.W ? pages : c.W;
}
static int select_chunks(int32_t width) { return (width + SELECT_CHUNK - 1) / SELECT_CHUNK; }
size_t paged_select_ws_bytes(const PagedCache& c, int32_t B, int32_t G, int32_t bound) {
  const int32_t width = select_width(c, bound);
  return (size_t)B * (size_t)G * ((size_t)width * sizeof(uint32_t) + (size_t)select_chunks(width) * SELECT_WAVES * sizeof(Extent));
}

void launch_paged_select(bool bf16, PagedSelectArgs a, void* ws, hipStream_t s) {
  a.width = select_width(a.c, a.bound);
  a.scores = (uint32_t*)ws;
  a.extents = a.scores + (size_t)a.B * a.G * a.width;
  const int64_t heads = (int64_t)a.B * a.G;
  const int chunks = select_chunks(a.width);
  auto most = [](int64_t n, int64_t limit) { return (unsigned)(n < limit ? n : limit); };
  const dim3 each(most(a.G, 4096), (unsigned)a.B), wg(SELECT_THREADS);
  // One launch, a workgroup for each entry and head, or two, the first on the whole chip.  Us, one / two launches (1 query, from 64 heads on 4): 8 heads of
  // 242 pages 9.8 / 10.6, of 492 11.5 / 10.2, of 1992 26.5 / 14.4; 32 heads of 367 pages 10.9 / 10.9, of 1992 27.9 / 21.1; 64 heads of 1992 28.4 / 27.8, 80
  // 28.4 / 30.7, 96 28.6 / 32.9, 256 50.9 / 72.8, 264 72.6 / 74.3; 256 of up to 304 13.1 / 20.1.
  if (a.width <= SELECT_HELD && heads < (1 << 30) && (heads >= 72 || a.width <= 256)) {
    ProfScope ps("paged_select", s);
    if (bf16) hipLaunchKernelGGL((paged_select_kernel<true>), dim3(most((heads + 7) / 8 * 8, 65536)), wg, 0, s, a);
    else hipLaunchKernelGGL((paged_select_kernel<false>), dim3(most((heads + 7) / 8 * 8, 65536)), wg, 0, s, a);
    return;
  }
  {
    ProfScope ps("paged_score", s);
    const dim3 all(most(chunks, 1024), most(a.G, 256), (unsigned)a.B);
    if (bf16) hipLaunchKernelGGL((paged_score_kernel<true>), all, wg, 0, s, a, chunks);
    else hipLaunchKernelGGL((paged_score_kernel<false>), all, wg, 0, s, a, chunks);
  }
  ProfScope ps("paged_pick", s);
  if (bf16) hipLaunchKernelGGL((paged_pick_kernel<true>), each, wg, 0, s, a, chunks);
  else hipLaunchKernelGGL((paged_pick_kernel<false>), each, wg, 0, s, a, chunks);
}

}  // namespace beagle
