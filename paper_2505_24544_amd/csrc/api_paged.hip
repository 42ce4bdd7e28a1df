// C-ABI entry points of the paged cache: validation, workspace carving and launch order only.
#include "api_internal.h"
#include "paged.h"
#include "proj_rows.h"

#include <math.h>
#include <string.h>

using namespace beagle;
using namespace beagle::detail;

namespace beagle {
namespace {

struct Paged {
  Dims d;                                  // of desc; projections: Tq rows in all
  PagedCache c;
  int64_t page_bytes;                      // K (or V) of one page
  double scale;                            // the definition's, not rounded to float
};

beagle_status check_cache(const beagle_paged_cache* p, PagedCache* c) {
  if (!p) return BEAGLE_ERR_NULL;
  if (p->struct_size != (int32_t)sizeof(beagle_paged_cache) || p->reserved != 0) return BEAGLE_ERR_SHAPE;
  if (p->n_pages < 1 || p->page_rows < 1 || p->n_slots < 1 || p->slot_pages < 1) return BEAGLE_ERR_SHAPE;
  // the kernels divide by the page's rows with a shift, and keep four neighbouring rows on one page
  if (p->page_rows < 4 || p->page_rows > 4096 || (p->page_rows & (p->page_rows - 1))) return BEAGLE_ERR_UNSUPPORTED;
  // row numbers and sums of blocks over 64 sequences stay within int32
  if ((int64_t)p->slot_pages * p->page_rows > (1 << 28) || p->n_pages > (1 << 28) || p->n_slots > PAGED_MAX_BATCH)
    return BEAGLE_ERR_UNSUPPORTED;
  const void* ptrs[] = {p->k_pages, p->v_pages, p->page_table, p->lens, p->refs};
  for (const void* q : ptrs) if (!q) return BEAGLE_ERR_NULL;
  if (!aligned16(p->k_pages) || !aligned16(p->v_pages)) return BEAGLE_ERR_ALIGN;
  if ((((uintptr_t)p->page_table) | ((uintptr_t)p->lens) | ((uintptr_t)p->refs)) & 3u) return BEAGLE_ERR_ALIGN;
  c->k = p->k_pages; c->v = p->v_pages; c->table = p->page_table; c->lens = p->lens; c->refs = p->refs;
  c->P = p->n_pages; c->N = p->n_slots; c->W = p->slot_pages;
  c->shift = __builtin_ctz((unsigned)p->page_rows);
  return BEAGLE_OK;
}

// states: the call projects states of width D, so D and the products' operand limits count
beagle_status check_paged(const beagle_xattn_desc* desc, const beagle_paged_cache* cache, bool states, Paged* out) {
  if (!desc) return BEAGLE_ERR_NULL;
  if (desc->struct_size != (int32_t)sizeof(beagle_xattn_desc)) return BEAGLE_ERR_SHAPE;
  if (desc->batch < 1 || desc->seq_q < 1 || desc->seq_kv < 1) return BEAGLE_ERR_SHAPE;
  if (desc->batch > PAGED_MAX_BATCH || (int64_t)desc->batch * desc->seq_q > (1 << 24)) return BEAGLE_ERR_UNSUPPORTED;
  if (desc->flags & ~(uint32_t)BEAGLE_FLAG_ROPE) return BEAGLE_ERR_UNSUPPORTED;
  // the remaining checks are those of the draft step on all rows of the call as one batch entry
  beagle_xattn_desc one = *desc;
  one.batch = 1;
  one.seq_q = states ? desc->batch * desc->seq_q : 1;
  one.seq_kv = 1;
  if (!states) one.hidden = 64;            // (not read)
  beagle_status st = check_desc(&one, true, &out->d);
  if (st != BEAGLE_OK) return st;
  Dims& d = out->d;
  d.B = desc->batch; d.S = desc->seq_q; d.L = desc->seq_kv; d.Tq = d.B * d.S;
  out->scale = desc->softmax_scale > 0.f ? (double)desc->softmax_scale : 1.0 / sqrt((double)d.d);
  // grids of less than 2^32 threads a side
  const int64_t rows = d.S * (d.H / d.G);
  if (rows > (1 << 24) || d.G * ((rows + 15) / 16) > (1 << 24) || d.H * d.S > (1 << 24)) return BEAGLE_ERR_UNSUPPORTED;
  st = check_cache(cache, &out->c);
  if (st != BEAGLE_OK) return st;
  out->page_bytes = ((int64_t)1 << out->c.shift) * d.GD * (int64_t)d.esz;
  return BEAGLE_OK;
}

// workspaces of the calls on states: the projected rows, then what the projections and the paged call themselves need
struct StepWs { size_t a, b, pos, angles, proj, call, total; };
size_t proj_bytes(const Dims& d, int64_t n, int64_t N, int64_t K, bool pair) {
  if (!d.bf16 || !kv_append_bf16_fits((int32_t)n, (int32_t)N, (int32_t)K)) return 0;
  return align_up(kv_append_bf16_ws_bytes((int32_t)n, (int32_t)N, (int32_t)K)) / (pair ? 1 : 2);
}
// Rotated bf16 queries of up to this many rows are projected in passes of PROJ_ROWS, whose float sums are rotated; more are one tiled product that
// is stored and rotated in place, as in the training forward, so they round twice.  A draft step at 4096 channels, us, in passes / by the
// product: 65 rows 128 / 139, 120 87 / 84, 128 82 / 78, 192 96 / 78, 512 183 / 88.
constexpr int64_t ROTATED_ROWS = 2 * PROJ_ROWS;
int64_t pass_rows(const Dims& d) { return d.Tq < PROJ_ROWS ? d.Tq : PROJ_ROWS; }
bool rotates_sums(const Dims& d) {
  return d.rope && d.bf16 && d.Tq <= ROTATED_ROWS && kv_append_bf16_fits((int32_t)pass_rows(d), (int32_t)d.HD, (int32_t)d.D);
}
size_t larger(size_t a, size_t b) { return a > b ? a : b; }
StepWs draft_layout(const Dims& d) {
  StepWs w; size_t o = 0;
  w.a = o; o += align_up((size_t)(d.Tq * d.HD) * d.esz);       // q
  w.b = o; o += align_up((size_t)(d.Tq * d.HD) * d.esz);       // o
  w.pos = o; o += align_up((size_t)d.Tq * sizeof(int32_t));
  w.angles = o; if (rotates_sums(d)) o += align_up((size_t)pass_rows(d) * 64 * sizeof(float2));
  w.proj = o; o += align_up(larger(proj_bytes(d, rotates_sums(d) ? pass_rows(d) : d.Tq, d.HD, d.D, false), proj_bytes(d, d.Tq, d.D, d.HD, false)));
  w.call = o; o += align_up(paged_attn_ws_bytes((int32_t)d.B, (int32_t)d.S, (int32_t)d.H, (int32_t)d.G));
  w.total = o;
  return w;
}
StepWs append_layout(const Dims& d, const PagedCache& c) {
  StepWs w; size_t o = 0;
  w.a = o; o += align_up((size_t)(d.Tq * d.GD) * d.esz);       // K rows
  w.b = o; o += align_up((size_t)(d.Tq * d.GD) * d.esz);       // V rows
  w.pos = w.angles = o;
  w.proj = o; o += proj_bytes(d, d.Tq, d.GD, d.D, true);
  w.call = o; o += align_up(paged_append_ws_bytes(c, (int32_t)d.B));
  w.total = o;
  return w;
}

PagedAttnArgs attn_of(const Paged& p) {
  PagedAttnArgs a; memset(&a, 0, sizeof(a));
  a.c = p.c;
  a.B = (int32_t)p.d.B; a.M = (int32_t)p.d.S; a.H = (int32_t)p.d.H; a.G = (int32_t)p.d.G; a.d = (int32_t)p.d.d;
  const int64_t most = (int64_t)p.c.W << p.c.shift;
  a.bound = (int32_t)(p.d.L < most ? p.d.L : most);
  a.scale = p.scale;
  return a;
}
PagedAppendArgs append_of(const Paged& p) {
  PagedAppendArgs a; memset(&a, 0, sizeof(a));
  a.c = p.c;
  a.B = (int32_t)p.d.B; a.M = (int32_t)p.d.S; a.G = (int32_t)p.d.G; a.d = (int32_t)p.d.d;
  a.rope = p.d.rope ? 1 : 0; a.l2base = p.d.rope ? log2((double)p.d.rope_base) : 0.0; a.rope_pos = p.d.rope_pos;
  return a;
}

beagle_status check_view(const int32_t* slots, const int32_t* n_true, const uint32_t* tree_mask, int32_t mask_words,
                         int32_t window, int32_t sinks) {
  if (window < 0 || window > (1 << 28) || sinks < 0 || sinks > (1 << 28) || mask_words < 0) return BEAGLE_ERR_SHAPE;
  if (mask_words > 0 && !tree_mask) return BEAGLE_ERR_NULL;
  if ((((uintptr_t)slots) | ((uintptr_t)n_true) | ((uintptr_t)tree_mask)) & 3u) return BEAGLE_ERR_ALIGN;
  return BEAGLE_OK;
}
void set_view(PagedAttnArgs& a, const int32_t* slots, const int32_t* n_true, const uint32_t* tree_mask, int32_t mask_words,
              int32_t window, int32_t sinks) {
  a.slots = slots; a.n_true = n_true;
  a.tree = tree_mask; a.words = tree_mask ? mask_words : 0;
  a.window = window; a.sinks = sinks;
}
bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

}  // namespace
}  // namespace beagle

size_t beagle_xattn_paged_workspace_bytes(const beagle_xattn_desc* desc, const beagle_paged_cache* cache, int which) {
  Paged p;
  if (check_paged(desc, cache, which == BEAGLE_WS_PAGED_DRAFT || which == BEAGLE_WS_PAGED_KV_APPEND, &p) != BEAGLE_OK) return 0;
  switch (which) {
    case BEAGLE_WS_PAGED_ATTEND: return align_up(paged_attn_ws_bytes((int32_t)p.d.B, (int32_t)p.d.S, (int32_t)p.d.H, (int32_t)p.d.G));
    case BEAGLE_WS_PAGED_APPEND: return align_up(paged_append_ws_bytes(p.c, (int32_t)p.d.B));
    case BEAGLE_WS_PAGED_FORK: return align_up(paged_fork_ws_bytes(p.c, (int32_t)p.d.B));
    case BEAGLE_WS_PAGED_COMPACT: return align_up(paged_compact_ws_bytes(p.c));
    case BEAGLE_WS_PAGED_DRAFT: return draft_layout(p.d).total;
    case BEAGLE_WS_PAGED_KV_APPEND: return append_layout(p.d, p.c).total;
    default: return 0;
  }
}

namespace {
beagle_status check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (!workspace) return BEAGLE_ERR_NULL;
  if (((uintptr_t)workspace) % WS_ALIGN) return BEAGLE_ERR_ALIGN;
  return bytes < need ? BEAGLE_ERR_WORKSPACE : BEAGLE_OK;
}
}  // namespace

beagle_status beagle_xattn_paged_attend(const beagle_xattn_desc* desc, const beagle_paged_cache* cache, const void* q,
    const int32_t* slots, const int32_t* n_true, const uint32_t* tree_mask, int32_t mask_words, int32_t window, int32_t sinks,
    void* o, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Paged p; beagle_status st = check_paged(desc, cache, false, &p);
  if (st != BEAGLE_OK) return st;
  if (!q || !o || !lse) return BEAGLE_ERR_NULL;
  if (!aligned16(q) || !aligned16(o) || !aligned16(lse)) return BEAGLE_ERR_ALIGN;
  st = check_view(slots, n_true, tree_mask, mask_words, window, sinks);
  if (st != BEAGLE_OK) return st;
  st = check_workspace(workspace, workspace_bytes, beagle_xattn_paged_workspace_bytes(desc, cache, BEAGLE_WS_PAGED_ATTEND));
  if (st != BEAGLE_OK) return st;
  (void)hipGetLastError();
  PagedAttnArgs a = attn_of(p);
  set_view(a, slots, n_true, tree_mask, mask_words, window, sinks);
  a.q = q; a.o = o; a.lse = lse;
  launch_paged_attn(p.d.bf16, a, workspace, (hipStream_t)hip_stream);
  return hip_status();
}

beagle_status beagle_xattn_paged_append(const beagle_xattn_desc* desc, const beagle_paged_cache* cache, const int32_t* slots,
    const int32_t* pos, const int32_t* n_new, const void* k_new, const void* v_new, int32_t* short_pages,
    void* workspace, size_t workspace_bytes, void* hip_stream) {
  Paged p; beagle_status st = check_paged(desc, cache, false, &p);
  if (st != BEAGLE_OK) return st;
  if (!k_new || !v_new) return BEAGLE_ERR_NULL;
  if (!aligned16(k_new) || !aligned16(v_new)) return BEAGLE_ERR_ALIGN;
  if ((((uintptr_t)slots) | ((uintptr_t)pos) | ((uintptr_t)n_new) | ((uintptr_t)short_pages)) & 3u) return BEAGLE_ERR_ALIGN;
  st = check_workspace(workspace, workspace_bytes, beagle_xattn_paged_workspace_bytes(desc, cache, BEAGLE_WS_PAGED_APPEND));
  if (st != BEAGLE_OK) return st;
  (void)hipGetLastError();
  PagedAppendArgs a = append_of(p);
  a.slots = slots; a.pos = pos; a.n_new = n_new; a.k_new = k_new; a.v_new = v_new; a.short_pages = short_pages;
  launch_paged_append(p.d.bf16, a, workspace, (hipStream_t)hip_stream);
  return hip_status();
}

beagle_status beagle_xattn_paged_fork(const beagle_xattn_desc* desc, const beagle_paged_cache* cache, const int32_t* dst,
    const int32_t* src, const int32_t* rows, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Paged p; beagle_status st = check_paged(desc, cache, false, &p);
  if (st != BEAGLE_OK) return st;
  if (!dst || !src) return BEAGLE_ERR_NULL;
  if ((((uintptr_t)dst) | ((uintptr_t)src) | ((uintptr_t)rows)) & 3u) return BEAGLE_ERR_ALIGN;
  st = check_workspace(workspace, workspace_bytes, beagle_xattn_paged_workspace_bytes(desc, cache, BEAGLE_WS_PAGED_FORK));
  if (st != BEAGLE_OK) return st;
  (void)hipGetLastError();
  launch_paged_fork(p.c, dst, src, rows, (int32_t)p.d.B, workspace, (hipStream_t)hip_stream);
  return hip_status();
}

beagle_status beagle_xattn_paged_compact(const beagle_xattn_desc* desc, const beagle_paged_cache* cache,
    const beagle_paged_cache* into, int32_t* short_pages, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Paged p; beagle_status st = check_paged(desc, cache, false, &p);
  if (st != BEAGLE_OK) return st;
  PagedCache to;
  st = check_cache(into, &to);
  if (st != BEAGLE_OK) return st;
  if (to.shift != p.c.shift || to.N != p.c.N) return BEAGLE_ERR_SHAPE;
  if (((uintptr_t)short_pages) & 3u) return BEAGLE_ERR_ALIGN;
  // every array of the target is written while the source's are read
  const struct { const void* p; int64_t n; } from_[] = {
      {p.c.k, p.c.P * p.page_bytes}, {p.c.v, p.c.P * p.page_bytes}, {p.c.table, (int64_t)p.c.N * p.c.W * 4}, {p.c.lens, (int64_t)p.c.N * 4},
      {p.c.refs, (int64_t)p.c.P * 4}}, to_[] = {
      {to.k, to.P * p.page_bytes}, {to.v, to.P * p.page_bytes}, {to.table, (int64_t)to.N * to.W * 4}, {to.lens, (int64_t)to.N * 4},
      {to.refs, (int64_t)to.P * 4}};
  for (const auto& x : from_) for (const auto& y : to_) if (overlap(x.p, x.n, y.p, y.n)) return BEAGLE_ERR_SHAPE;
  st = check_workspace(workspace, workspace_bytes, beagle_xattn_paged_workspace_bytes(desc, cache, BEAGLE_WS_PAGED_COMPACT));
  if (st != BEAGLE_OK) return st;
  (void)hipGetLastError();
  launch_paged_compact(p.c, to, p.page_bytes, short_pages, workspace, (hipStream_t)hip_stream);
  return hip_status();
}

namespace {
// y = x W: a handful of rows stream W split over k, more take the tiled product
void project(const Dims& d, const void* x, const void* w, void* y, int64_t N, int64_t K, void* ws, const char* name, hipStream_t s) {
  if (d.bf16 && kv_append_bf16_fits((int32_t)d.Tq, (int32_t)N, (int32_t)K))
    launch_proj_rows_bf16(x, w, y, (int32_t)d.Tq, (int32_t)N, (int32_t)K, ws, name, s);
  else
    run_gemm(d, group1(gemm_nn(x, w, y, d.Tq, N, K)), s, name);
}
}  // namespace

beagle_status beagle_xattn_draft_step_paged(const beagle_xattn_desc* desc, const beagle_paged_cache* cache, const void* x_draft,
    const void* wq, const void* wo, const int32_t* slots, const int32_t* n_true, const uint32_t* tree_mask, int32_t mask_words,
    int32_t window, int32_t sinks, void* y, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Paged p; beagle_status st = check_paged(desc, cache, true, &p);
  if (st != BEAGLE_OK) return st;
  const void* ptrs[] = {x_draft, wq, wo, y, lse};
  for (const void* q : ptrs) if (!q) return BEAGLE_ERR_NULL;
  for (const void* q : ptrs) if (!aligned16(q)) return BEAGLE_ERR_ALIGN;
  st = check_view(slots, n_true, tree_mask, mask_words, window, sinks);
  if (st != BEAGLE_OK) return st;
  const Dims& d = p.d;
  const StepWs w = draft_layout(d);
  st = check_workspace(workspace, workspace_bytes, w.total);
  if (st != BEAGLE_OK) return st;
  hipStream_t s = (hipStream_t)hip_stream;
  (void)hipGetLastError();
  char* base = (char*)workspace;
  const int32_t* at = d.rope_pos;
  if (d.rope && !at) {
    launch_paged_positions(p.c, slots, (int32_t)d.B, (int32_t)d.S, (int32_t*)(base + w.pos), s);
    at = (const int32_t*)(base + w.pos);
  }
  if (rotates_sums(d)) {
    for (int64_t r = 0; r < d.Tq; r += PROJ_ROWS) {
      const int64_t n = d.Tq - r < PROJ_ROWS ? d.Tq - r : PROJ_ROWS;
      const RopeRows rope = {at + r, 0, log2((double)d.rope_base), (float2*)(base + w.angles), 1};
      launch_proj_rope_rows_bf16((const bf16_t*)x_draft + r * d.D, wq, (bf16_t*)(base + w.a) + r * d.HD, (int32_t)n, (int32_t)d.HD, (int32_t)d.D,
                                 base + w.proj, rope, "draft_proj_q", s);
    }
  } else {
    project(d, x_draft, wq, base + w.a, d.HD, d.D, base + w.proj, "draft_proj_q", s);
    if (d.rope) {
      RopeArgs r = rope_args(d, false);
      rope_add(r, base + w.a, d.Tq, d.Tq, d.H, 0, at);
      launch_rope(d.bf16, r, s, "draft_rope_q");
    }
  }
  PagedAttnArgs a = attn_of(p);
  set_view(a, slots, n_true, tree_mask, mask_words, window, sinks);
  a.q = base + w.a; a.o = base + w.b; a.lse = lse;
  launch_paged_attn(d.bf16, a, base + w.call, s);
  project(d, base + w.b, wo, y, d.D, d.HD, base + w.proj, "draft_proj_out", s);
  return hip_status();
}

beagle_status beagle_xattn_kv_append_paged(const beagle_xattn_desc* desc, const beagle_paged_cache* cache, const void* x_new,
    const void* wk, const void* wv, const int32_t* slots, const int32_t* pos, const int32_t* n_new, int32_t* short_pages,
    void* workspace, size_t workspace_bytes, void* hip_stream) {
  Paged p; beagle_status st = check_paged(desc, cache, true, &p);
  if (st != BEAGLE_OK) return st;
  const void* ptrs[] = {x_new, wk, wv};
  for (const void* q : ptrs) if (!q) return BEAGLE_ERR_NULL;
  for (const void* q : ptrs) if (!aligned16(q)) return BEAGLE_ERR_ALIGN;
  if ((((uintptr_t)slots) | ((uintptr_t)pos) | ((uintptr_t)n_new) | ((uintptr_t)short_pages)) & 3u) return BEAGLE_ERR_ALIGN;
  const Dims& d = p.d;
  const StepWs w = append_layout(d, p.c);
  st = check_workspace(workspace, workspace_bytes, w.total);
  if (st != BEAGLE_OK) return st;
  hipStream_t s = (hipStream_t)hip_stream;
  (void)hipGetLastError();
  char* base = (char*)workspace;
  if (d.bf16 && kv_append_bf16_fits((int32_t)d.Tq, (int32_t)d.GD, (int32_t)d.D)) {
    launch_kv_append_bf16(x_new, wk, wv, base + w.a, base + w.b, (int32_t)d.Tq, (int32_t)d.GD, (int32_t)d.D, base + w.proj, s);
  } else {
    GemmGroup g; memset(&g, 0, sizeof(g));
    g.count = 2;
    g.p[0] = gemm_nn(x_new, wk, base + w.a, d.Tq, d.GD, d.D);
    g.p[1] = gemm_nn(x_new, wv, base + w.b, d.Tq, d.GD, d.D);
    run_gemm(d, g, s, "kv_append");
  }
  PagedAppendArgs a = append_of(p);
  a.slots = slots; a.pos = pos; a.n_new = n_new; a.k_new = base + w.a; a.v_new = base + w.b; a.short_pages = short_pages;
  launch_paged_append(d.bf16, a, base + w.call, s);
  return hip_status();
}
