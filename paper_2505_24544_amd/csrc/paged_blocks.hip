// Attention to a few pages of a long context: bounds of every page's keys, the pages that they put first, attention over those.
//
//   lo_pc = min_j k_jc, hi_pc = max_j k_jc over the rows j of page p;   score_p = max_r sum_c max(q_rc lo_pc, q_rc hi_pc),
//
// which no <q_r, k_j> of the page exceeds.  An entry's first pages and its last ones are always seen; of those between them a kv
// head sees the n_select with the highest scores.
#include "paged_attend.h"

namespace beagle {
namespace {

// ------------------------------------------------------------------ bounds
// One workgroup for a page and 64 pieces of 16 bytes of its rows; the waves take the rows in turns.
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
struct Span { int lead, count; const int32_t* table; };
// the pages that an entry's selection is made of: `count` of them from `lead` on
__device__ __forceinline__ Span span_of(const PagedSelectArgs& a, int b) {
  const int slot = paged_slot(a.c, a.slots, b);
  const int n = min(paged_len(a.c, slot), a.bound);
  const PagedPick p = paged_pick(n, a.n_true ? a.n_true[b] : INT32_MAX, a.window, a.sinks, a.n_select, a.c.shift);
  return {p.lead, p.listed + p.gap, a.c.table + (int64_t)max(slot, 0) * a.c.W};
}

// Scores.  Sixteen lanes take a page; what they add up is exact in 64 bits but for the last of them (a product of two bf16 has 16 bits, of two
// floats 48), so that the order of the pages is that of the definition.  It is rounded to float once.
constexpr int SELECT_PAGES = 64, SELECT_ROWS = 16;           // pages of a workgroup, query rows that are held at a time
template <bool BF16>
__global__ __launch_bounds__(256) void paged_score_kernel(PagedSelectArgs a, int64_t units, int chunks) {
  constexpr int E = BF16 ? 2 : 4, N = 8;
  __shared__ float sq[SELECT_ROWS][128];
  const int rep = a.H / a.G, R = a.M * rep;
  const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int chunk = (int)(u % chunks);
    const int64_t bg = u / chunks;
    const int b = (int)(bg / a.G), g = (int)(bg % a.G);
    const Span span = span_of(a, b);
    if (span.count <= a.n_select || chunk * SELECT_PAGES >= span.count) continue;      // (the same in all lanes)
    constexpr int EACH = SELECT_PAGES / 16;
    float lo[EACH][N], hi[EACH][N], best[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int i = chunk * SELECT_PAGES + e * 16 + group;
      const int page = i < span.count ? span.table[span.lead + i] : -1;
      const bool there = (unsigned)page < (unsigned)a.c.P;
      best[e] = -INFINITY;
      const addr_t src = (addr_t)a.bounds + ((int64_t)(there ? page : 0) * a.G + g) * 2 * a.d * E;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int ch = lane * N + i;
          float v = 0.f;
          if (ch < a.d) {
            if constexpr (BF16) v = bf16_to_f32(((const bf16_t*)src)[h * a.d + ch]);
            else v = ((const float*)src)[h * a.d + ch];
          }
          (h ? hi : lo)[e][i] = v;
        }
      if (!there) best[e] = NAN;
    }
    for (int r0 = 0; r0 < R; r0 += SELECT_ROWS) {
      __syncthreads();
      for (int i = threadIdx.x; i < SELECT_ROWS * 128; i += 256) {
        const int r = r0 + i / 128, ch = i % 128;
        float v = 0.f;
        if (r < R && ch < a.d) {
          const int64_t at = (((int64_t)b * a.M + r / rep) * a.H + g * rep + r % rep) * a.d + ch;
          v = BF16 ? bf16_to_f32(((const bf16_t*)a.q)[at]) : ((const float*)a.q)[at];
        }
        sq[i / 128][ch] = v;
      }
      __syncthreads();
      for (int r = 0; r < min(SELECT_ROWS, R - r0); ++r) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
          double s = 0.0;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float q = sq[r][lane * N + i], x = q > 0.f ? hi[e][i] : q < 0.f ? lo[e][i] : 0.f;
            s = fma((double)(q == q ? q : 0.f), (double)x, s);
          }
#pragma unroll
          for (int i = 1; i < 16; i *= 2) s += __shfl_xor(s, i);
          best[e] = isnan(best[e]) ? best[e] : fmaxf(best[e], (float)s);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int i = chunk * SELECT_PAGES + e * 16 + group;
      if (lane == 0 && i < span.count) a.scores[bg * a.width + i] = isnan(best[e]) ? -INFINITY : best[e] + 0.f;
    }
    __syncthreads();
  }
}

// larger scores have larger keys
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// The n_select largest of an entry's and head's scores: the key of the last of them is found eight bits at a time, then the pages are
// written in order, of those with that key the first ones.
__global__ __launch_bounds__(256) void paged_pick_kernel(PagedSelectArgs a) {
  __shared__ uint32_t count[256], state[2];
  __shared__ int above[4], level[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int64_t bg = blockIdx.x; bg < (int64_t)a.B * a.G; bg += gridDim.x) {
    const Span span = span_of(a, (int)(bg / a.G));
    int32_t* out = a.pages + bg * a.n_select;
    if (span.count <= a.n_select) {
      for (int i = tid; i < a.n_select; i += 256) out[i] = i < span.count ? span.lead + i : -1;
      continue;
    }
    const float* scores = a.scores + bg * a.width;
    uint32_t prefix = 0, want = a.n_select;                  // keys with these leading bits; how many of them are picked
    for (int shift = 24; shift >= 0; shift -= 8) {
      count[tid] = 0;
      __syncthreads();
      for (int i = tid; i < span.count; i += 256) {
        const uint32_t k = key_of(scores[i]);
        if (shift == 24 || k >> (shift + 8) == prefix) atomicAdd(&count[k >> shift & 255], 1u);
      }
      __syncthreads();
      if (wave == 0) {                                       // from the largest bin down: four bins to a lane
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) { c[i] = count[255 - 4 * lane - i]; sum += c[i]; }
        uint32_t before = (uint32_t)sum_upto((int)sum) - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < want && want <= before + c[i]) { state[0] = prefix << 8 | (uint32_t)(255 - 4 * lane - i); state[1] = want - before; }
          before += c[i];
        }
      }
      __syncthreads();
      prefix = state[0]; want = state[1];
      __syncthreads();
    }
    int written = 0, taken = 0;                              // of the pages before: picked, and those of them with the last key
    for (int i0 = 0; i0 < span.count; i0 += 256) {
      const uint32_t k = i0 + tid < span.count ? key_of(scores[i0 + tid]) : 0;
      const bool in = i0 + tid < span.count;
      const unsigned long long gt = __ballot(in && k > prefix), eq = __ballot(in && k == prefix), lower = (1ull << lane) - 1;
      if (lane == 0) { above[wave] = __popcll(gt); level[wave] = __popcll(eq); }
      __syncthreads();
      int ties = taken, at = written;
      for (int w = 0; w < wave; ++w) { at += above[w] + min(level[w], max((int)want - ties, 0)); ties += level[w]; }
      const int tie = ties + __popcll(eq & lower);
      at += __popcll(gt & lower) + max(min(tie, (int)want) - min(ties, (int)want), 0);
      if (in && (k > prefix || (k == prefix && tie < (int)want))) out[at] = span.lead + i0 + tid;
      for (int w = 0; w < 4; ++w) { written += above[w] + min(level[w], max((int)want - taken, 0)); taken += level[w]; }
      __syncthreads();
    }
  }
}

}  // namespace

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
size_t paged_select_ws_bytes(const PagedCache& c, int32_t B, int32_t G, int32_t bound) {
  return (size_t)B * (size_t)G * (size_t)select_width(c, bound) * sizeof(float);
}

void launch_paged_select(bool bf16, PagedSelectArgs a, void* ws, hipStream_t s) {
  a.scores = (float*)ws;
  a.width = select_width(a.c, a.bound);
  if (a.width > a.n_select) {                                // (otherwise every page is picked)
    ProfScope ps("paged_score", s);
    const int chunks = (a.width + SELECT_PAGES - 1) / SELECT_PAGES;
    const int64_t units = (int64_t)a.B * a.G * chunks;
    const dim3 grid((unsigned)(units < 8192 ? units : 8192));
    if (bf16) hipLaunchKernelGGL((paged_score_kernel<true>), grid, dim3(256), 0, s, a, units, chunks);
    else hipLaunchKernelGGL((paged_score_kernel<false>), grid, dim3(256), 0, s, a, units, chunks);
  }
  ProfScope ps("paged_pick", s);
  const int64_t heads = (int64_t)a.B * a.G;
  hipLaunchKernelGGL(paged_pick_kernel, dim3((unsigned)(heads < 65536 ? heads : 65536)), dim3(256), 0, s, a);
}

}  // namespace beagle
