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
    total += blocks;
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
      u.b = b0 + l;
      u.units = __shfl(mine, l);
      u.i = want_entry ? 0 : which - base - (__shfl(upto, l) - u.units);
      u.first = parts + __shfl(pupto, l) - (u.units > 1 ? u.units : 0);
      return u;
    }
    base += __shfl(upto, 63);
    parts += __shfl(pupto, 63);
  }
  return u;
}

__device__ __forceinline__ float max_over_keys(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
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
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4;
  // row blocks of one unit and head stand eight workgroups apart: on one XCD, whose L2 has the rows after the first
  const int id = blockIdx.x, ug = id / (8 * rowblocks) * 8 + id % 8, rb = id / 8 % rowblocks;
  if (ug >= heads8) return;
  const int head = ug % a.G;
  const Unit u = find_unit(a, ug / a.G, false);
  if (u.b < 0) return;
  const int slot = paged_slot(a.c, a.slots, u.b);
  const PagedRows rows = rows_of(a, slot, u.b);
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
  const float c2 = a.scale * LOG2E;

  auto page_of = [&](int row) { return paged_page(table, row, paged_seen(rows, row), a.c.shift, a.c.P); };
  for (int vb = first + wave; vb < last; vb += WAVES) {
    const int block = paged_block(rows, vb);
#pragma unroll
    for (int sub = 0; sub < PAGED_BLOCK / S::KROWS; ++sub) {
      const int base = block * PAGED_BLOCK + sub * S::KROWS;
      if (base >= rows.n) break;
      // ---- K rows, one in each lane's l16; V rows, four neighbours (one page: its rows are a multiple of four)
      u32x4 k[S::KT][S::NJ], v[S::NV][NH];
#pragma unroll
      for (int t = 0; t < S::KT; ++t) {
        const int row = base + 16 * t + l16, p = page_of(row);
        const char* src = p >= 0 ? kbase + (((int64_t)p << a.c.shift) + (row & in_page)) * row_bytes : (const char*)zero_row;
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) {
          const int piece = (4 * j + g4) * 16;
          k[t][j] = *(const u32x4*)(BF16 || piece < a.d * E ? src + piece : (const char*)zero_row);
        }
      }
      bool seen[S::KT][4];
#pragma unroll
      for (int t = 0; t < S::KT; ++t) {
        const int r0 = base + 16 * t + 4 * g4;
        // (a page number that is not one hides its rows)
        const int p = paged_page(table, r0, r0 < rows.n, a.c.shift, a.c.P);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          seen[t][i] = p >= 0 && paged_seen(rows, r0 + i);
          const char* src = seen[t][i] ? vbase + (((int64_t)p << a.c.shift) + ((r0 + i) & in_page)) * row_bytes : (const char*)zero_row;
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            const int piece = (16 * h + l16) * 16;
            v[4 * t + i][h] = *(const u32x4*)(BF16 || piece < a.d * E ? src + piece : (const char*)zero_row);
          }
        }
      }
      // A drafted row that only some queries see may hold what is no number, which the others must not meet (0 * NaN is
      // NaN).  The matrix instructions mix all rows into all queries, so such a step adds row by row where it is seen.
      [[maybe_unused]] bool odd = false;
      if constexpr (TREE)
        if (base + S::KROWS > rows.nt) {
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
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        // ---- scores
        f32x4 s[S::KT];
#pragma unroll
        for (int kt = 0; kt < S::KT; ++kt) {
          s[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < S::NJ; ++j) {
            if constexpr (BF16) s[kt] = mfma_bf16(k[kt][j], q[t][j], s[kt]);
            else
#pragma unroll
              for (int e = 0; e < 4; ++e) s[kt] = mfma_f32(__uint_as_float(k[kt][j][e]), __uint_as_float(q[t][j][e]), s[kt]);
          }
        }
        float top = -INFINITY;
        [[maybe_unused]] bool saw[S::KT][4];
#pragma unroll
        for (int kt = 0; kt < S::KT; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            bool see = seen[kt][i];
            if constexpr (TREE) {
              const int bit = base + 16 * kt + 4 * g4 + i - rows.nt;
              if (see && bit >= 0)
                see = qm[t] < a.M && (bit >> 5) < a.words &&
                      (a.tree[((int64_t)u.b * a.M + qm[t]) * a.words + (bit >> 5)] >> (bit & 31) & 1u);
            }
            s[kt][i] = see ? s[kt][i] * c2 : -INFINITY;
            if constexpr (TREE) saw[kt][i] = see;
            top = fmaxf(top, s[kt][i]);
          }
        // ---- running maximum and sum
        const float now = fmaxf(mx[t], max_over_keys(top)), safe = now == -INFINITY ? 0.f : now;
        const float shrink = exp2_fast(mx[t] - safe);
        mx[t] = now;
        float p[S::KT][4], add = 0.f;
#pragma unroll
        for (int kt = 0; kt < S::KT; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i) { p[kt][i] = exp2_fast(s[kt][i] - safe); add += p[kt][i]; }
        sum[t] = sum[t] * shrink + add;
#pragma unroll
        for (int c = 0; c < S::NA; ++c) acc[t][c] *= shrink;
        // ---- O^T += V^T P^T
        if constexpr (TREE) if (odd) {
          float* mine = part_o[wave][l16];       // (free until the end)
#pragma unroll
          for (int kt = 0; kt < S::KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[16 * kt + 4 * g4 + i] = saw[kt][i] ? p[kt][i] : -1.f;
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          for (int j = 0; j < S::KROWS; ++j) {
            const float w = mine[j];
            const int row = base + j, pg = page_of(row);
            if (w == -1.f || pg < 0) continue;
            const char* src = vbase + (((int64_t)pg << a.c.shift) + (row & in_page)) * row_bytes;
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
          continue;
        }
        if constexpr (BF16) {
          // a probability as two bf16 numbers, 16 bits in all: the matrix pipe has the time, and the rounding of one
          // would cost the output as much again as its own (2^-9)
          u32x4 hi, lo;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = p[i >> 1][2 * (i & 1)], y = p[i >> 1][2 * (i & 1) + 1];
            hi[i] = pack_bf16x2(x, y);
            lo[i] = pack_bf16x2(x - __uint_as_float(hi[i] << 16), y - __uint_as_float(hi[i] & 0xffff0000u));
          }
#pragma unroll
          for (int c = 0; c < 8; ++c) {       // channels 8 l16 + c
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              w[i] = __builtin_amdgcn_perm(v[2 * i + 1][0][c >> 1], v[2 * i][0][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
            acc[t][c] = mfma_bf16(w, hi, acc[t][c]);
            acc[t][c] = mfma_bf16(w, lo, acc[t][c]);
          }
        } else {
#pragma unroll
          for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int c = 0; c < 4; ++c)       // channels 64 h + 4 l16 + c
#pragma unroll
              for (int i = 0; i < 4; ++i)
                acc[t][4 * h + c] = mfma_f32(__uint_as_float(v[i][h][c]), p[0][i], acc[t][4 * h + c]);
        }
      }
    }
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
int row_tiles(int R) { return R <= 16 ? 1 : 2; }
int units_aimed(int R, int G) {
  const int per = G * ((R + 16 * row_tiles(R) - 1) / (16 * row_tiles(R)));
  return per < AIM ? AIM / per : 1;
}

}  // namespace

// Partial sums: only entries of several units have them, and those are at most twice the units aimed at.
size_t paged_attn_ws_bytes(int32_t M, int32_t H, int32_t G) {
  const int64_t R = (int64_t)M * (H / G);
  return (size_t)2 * units_aimed((int)R, G) * G * R * (128 + 2) * sizeof(float);
}

void launch_paged_attn(bool bf16, PagedAttnArgs a, void* ws, hipStream_t s) {
  const int R = a.M * (a.H / a.G), RT = row_tiles(R), rowblocks = (R + 16 * RT - 1) / (16 * RT);
  a.target = units_aimed(R, a.G);
  a.least = WAVES;
  const int64_t rows = (int64_t)2 * a.target * a.G * R;
  a.part = (float*)ws;
  a.ml = a.part + rows * 128;
  const int heads8 = (a.target + a.B) * a.G;
  const dim3 grid((unsigned)((heads8 + 7) / 8 * 8 * rowblocks)), wg(64 * WAVES);
  const bool tree = a.n_true != nullptr, narrow = !bf16 && a.d <= 64;
  {
    ProfScope ps("paged_attn", s);
    auto go = [&](auto bf_, auto nh_) {
      constexpr bool BF = decltype(bf_)::value != 0;
      constexpr int NH = decltype(nh_)::value;
      if (RT == 1 && !tree) hipLaunchKernelGGL((paged_attn_kernel<BF, NH, 1, false>), grid, wg, 0, s, a, heads8, rowblocks);
      else if (RT == 1) hipLaunchKernelGGL((paged_attn_kernel<BF, NH, 1, true>), grid, wg, 0, s, a, heads8, rowblocks);
      else if (!tree) hipLaunchKernelGGL((paged_attn_kernel<BF, NH, 2, false>), grid, wg, 0, s, a, heads8, rowblocks);
      else hipLaunchKernelGGL((paged_attn_kernel<BF, NH, 2, true>), grid, wg, 0, s, a, heads8, rowblocks);
    };
    if (bf16) go(int_c<1>{}, int_c<1>{});
    else if (narrow) go(int_c<0>{}, int_c<1>{});
    else go(int_c<0>{}, int_c<2>{});
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
