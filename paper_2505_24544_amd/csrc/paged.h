// Key/value rows of many sequences in pages of one pool: what the launchers of paged_attn.hip and paged_pages.hip take,
// and the split of a batch's rows over workgroups.  Not part of the public interface.
#pragma once
#include "common.h"
#include "paged_index.h"

namespace beagle {

constexpr int PAGED_MAX_BATCH = 8192;      // entries of a call, and slots of a cache

// The caller's pool.  Whatever stands in the device arrays, no access leaves them: slot numbers, lengths and page
// numbers are checked where they are read.
struct PagedCache {
  void *k, *v;                             // [P, page_rows, G, d]
  int32_t *table, *lens, *refs;            // [N, W], [N], [P]
  int32_t P, shift, N, W;                  // page_rows == 1 << shift
};

struct PagedAttnArgs {
  PagedCache c;
  int32_t B, M, H, G, d;
  int32_t bound;                           // no sequence is taken to hold more rows
  double scale;
  float c2, c2_low;                        // scale * log2(e), set at the launch
  const void* q; void* o; float* lse;      // [B, M, H, d] x2, [B, H, M]
  const int32_t* slots;                    // [B] or null: entry b reads slot b
  const int32_t* n_true;                   // [B] or null: every row is a true one
  const uint32_t* tree; int32_t words;     // [B, M, words]
  int32_t window, sinks;                   // window 0: none
  const int32_t* lists; int32_t listed;    // [B, G, listed]: pages that a kv head sees besides (launch_paged_blocks)
  float* part; float* ml;                  // sums of the parts of entries that several workers share
  int2* parts;                             // [B] first worker of an entry, how many have a part of it
  int32_t target;                          // workers, at most
  bool long_runs;                          // see paged_split
};
size_t paged_attn_ws_bytes(int32_t B, int32_t M, int32_t H, int32_t G);
void launch_paged_attn(bool bf16, PagedAttnArgs a, void* ws, hipStream_t s);

void launch_paged_blocks(bool bf16, PagedAttnArgs a, void* ws, hipStream_t s);     // a.lists; workspace as launch_paged_attn's

// least and greatest value of every channel over the rows of a page
void launch_paged_bounds(bool bf16, const PagedCache& c, int32_t B, int32_t G, int32_t d, int32_t bound, const int32_t* slots,
                         const int32_t* first, void* bounds, hipStream_t s);

struct PagedSelectArgs {
  PagedCache c;
  int32_t B, M, H, G, d, bound;
  const void *q, *bounds;                  // [B, M, H, d], [P, G, 2, d]
  const int32_t *slots, *n_true;           // [B] or null
  int32_t window, sinks, n_select;
  int32_t* pages;                          // [B, G, n_select]
  uint32_t* scores; int32_t width;         // [B, G, width]: floats, then keys
  void* extents;                           // what they may be off by, the least and the greatest, chunk by chunk and wave by wave
};
size_t paged_select_ws_bytes(const PagedCache& c, int32_t B, int32_t G, int32_t bound);
void launch_paged_select(bool bf16, PagedSelectArgs a, void* ws, hipStream_t s);

// Entries group_first[g] .. group_first[g + 1] - 1 see the first n_shared[g] rows of the first of them
struct PagedSharedArgs {
  PagedAttnArgs a;                         // window 0
  const int32_t *group_first, *n_shared;   // [groups + 1], [groups]
  int32_t groups;
};
size_t paged_shared_ws_bytes(int32_t B, int32_t M, int32_t H, int32_t G);
void launch_paged_shared(bool bf16, PagedSharedArgs a, void* ws, hipStream_t s);

struct PagedAppendArgs {
  PagedCache c;
  int32_t B, M, G, d;
  const int32_t *slots, *pos, *n_new;      // [B] each, or null: slot b, behind the rows held, M
  const void *k_new, *v_new;               // [B, M, G, d]
  int32_t* short_pages;                    // [1]
  int32_t rope; double l2base;             // K rows are rotated at rope_pos[b * M + i], or at their row number
  const int32_t* rope_pos;
};
size_t paged_append_ws_bytes(const PagedCache& c, int32_t B);
void launch_paged_append(bool bf16, const PagedAppendArgs& a, void* ws, hipStream_t s);

// pos[b * M + m] = rows that entry b's sequence holds
void launch_paged_positions(const PagedCache& c, const int32_t* slots, int32_t B, int32_t M, int32_t* pos, hipStream_t s);

size_t paged_fork_ws_bytes(const PagedCache& c, int32_t B);
void launch_paged_fork(const PagedCache& c, const int32_t* dst, const int32_t* src, const int32_t* rows, int32_t B, void* ws,
                       hipStream_t s);

size_t paged_compact_ws_bytes(const PagedCache& c);
void launch_paged_compact(const PagedCache& from, const PagedCache& into, int64_t page_bytes, int32_t* short_pages, void* ws,
                          hipStream_t s);

// ---- read-side checks (device) ----
__device__ __forceinline__ int paged_slot(const PagedCache& c, const int32_t* slots, int b) { return paged_slot_of(slots ? slots[b] : b, c.N); }
__device__ __forceinline__ int paged_len(const PagedCache& c, int slot) { return slot < 0 ? 0 : paged_clamped(c.lens[slot], c.W, c.shift); }

// Inclusive sum over the lanes: within rows of 16, then what the rows before have.  All 64 lanes have to be active.
__device__ __forceinline__ int sum_upto(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);        // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);        // row_bcast 15, 31
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}
// Inclusive maximum over the lanes, of numbers from 0 on.
__device__ __forceinline__ int max_upto(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));
  return max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
}

}  // namespace beagle
