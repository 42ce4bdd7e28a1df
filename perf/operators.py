"""The paged cache and the attention that reads it, as cases that can be timed and checked.

A program that serves many users at once keeps the key/value rows of all their sequences in pages of one pool.  Per
iteration of speculative decoding it attends with a few draft queries of every sequence (`attend`), appends states behind
the true rows of every sequence (`append`), lets sequences branch (`fork`), and now and then moves the live pages into a
pool of another size (`compact`).

A case is a dict of plain values; `listed` names the standing ones, `draw` gives further ones of the same ranges.
`prepare` makes what the program holds before the call, `run` is one pass: the plain form in elementary torch operations,
or the library's calls where `own` is set.  `exact` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False

# (query heads, key/value heads) of the 7B-, the 8B- (grouped queries) and the 13B-shaped draft head, width 128
HEADS = ((32, 32), (32, 8), (40, 40))
# relatives of the fp32 reference problem: (query heads, key/value heads, head width)
HEADS_F32 = ((4, 4, 64), (4, 2, 64), (4, 4, 128), (8, 4, 64), (4, 4, 32))
ROPE_BASE = 10000.0


# ------------------------------------------------------------------ the cases
def _attend(batch, queries, rows, ragged, drafted, heads, kv_heads, page, window=0, sinks=0, dtype="bf16", head=128, name=None):
    c = dict(kind="attend", batch=batch, queries=queries, rows=rows, ragged=ragged, drafted=drafted, heads=heads,
             kv_heads=kv_heads, page=page, window=window, sinks=sinks, dtype=dtype, head=head)
    return dict(c, name=name) if name else c


def _append(batch, states, rows, ragged, kv_heads, page, dtype="bf16", head=128, name=None):
    c = dict(kind="append", batch=batch, states=states, rows=rows, ragged=ragged, kv_heads=kv_heads, page=page, dtype=dtype,
             head=head)
    return dict(c, name=name) if name else c


def _fork(batch, states, rows, ragged, kv_heads, page, dtype="bf16", head=128, name=None):
    c = dict(kind="fork", batch=batch, states=states, rows=rows, ragged=ragged, kv_heads=kv_heads, page=page, dtype=dtype,
             head=head)
    return dict(c, name=name) if name else c


def _compact(batch, rows, ragged, kv_heads, page, dtype="bf16", head=128, name=None):
    c = dict(kind="compact", batch=batch, rows=rows, ragged=ragged, kv_heads=kv_heads, page=page, dtype=dtype, head=head)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's short chat, one draft query: all launch latency
        _attend(1, 1, 777, False, 0, 32, 32, 16, name="attend_one_short"),
        # a batch of chats of different lengths with grouped queries, one query each: ordinary serving
        _attend(48, 1, 4096, True, 0, 32, 8, 16, name="attend_batch_8b"),
        # the paper's tree in a batch: ten queries of a depth under 50 drafted rows
        _attend(12, 10, 4096, True, 50, 32, 8, 32, name="attend_tree_8b"),
        # long contexts at the 13B shape: the largest
        _attend(4, 1, 32768, True, 0, 40, 40, 64, name="attend_long_13b"),
        # long streams of which a window and the first rows are attended
        _attend(32, 4, 20000, True, 0, 32, 8, 16, window=2048, sinks=4, name="window_batch_8b"),
        # the fp32 relative of the reference problem under a window: what is run to check a set-up
        _attend(6, 2, 1500, True, 0, 4, 2, 8, window=333, sinks=5, dtype="f32", head=64, name="window_f32"),
        # the accepted tokens of one iteration enter the caches of a batch
        _append(64, 5, 4000, True, 8, 16, name="append_accepted"),
        # prompts enter the cache
        _append(4, 1531, 500, True, 32, 64, name="append_prompts"),
        # a beam search's survivors take over their parents' rows
        _fork(24, 0, 3000, True, 8, 16, name="fork_beams"),
        # every branch of a sequence goes its own way: fork and first own rows, which copies the shared page
        _fork(32, 3, 1000, True, 32, 32, name="fork_branches"),
        # a pool of a few sequences, in fp32, moves
        _compact(8, 400, True, 4, 16, dtype="f32", head=64, name="compact_small"),
        # a half-empty pool is given back
        _compact(32, 6000, True, 8, 64, name="compact_pool"),
    ]


def _between(rng, lo, hi):
    """A whole number in [lo, hi], evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "attend", "window", "window", "append", "append", "fork", "compact"))
    f32 = rng.random() < 0.25
    heads, kv_heads, head = rng.choice(HEADS_F32) if f32 else rng.choice(HEADS) + (128,)
    dtype, page, ragged = "f32" if f32 else "bf16", rng.choice((8, 16, 16, 32, 64, 128)), rng.random() < 0.7
    if kind in ("attend", "window"):
        batch = _between(rng, 1, 96)
        # no more rows in all than the largest listed case has
        most = (20000 if f32 else 81920 * 40 // kv_heads) // batch
        rows = _between(rng, 1 if kind == "attend" else 40, max(2, min(32768, most)))
        queries = rng.choice((1, 1, 1, 2, 4, 7, 10, 16))
        if kind == "window":
            return _attend(batch, queries, rows, ragged, 0, heads, kv_heads, page, window=_between(rng, 16, 4096),
                           sinks=rng.choice((0, 1, 4, 4, 16, 100)), dtype=dtype, head=head)
        return _attend(batch, queries, rows, ragged, rng.choice((0, 0, rng.randint(1, 60))) if queries > 1 else 0, heads, kv_heads,
                       page, dtype=dtype, head=head)
    if kind == "append":
        batch = _between(rng, 1, 96)
        states = _between(rng, 1, max(1, min(4096, 8192 // batch)))
        return _append(batch, states, _between(rng, 1, max(2, 60000 // batch)), ragged, kv_heads, page, dtype, head)
    if kind == "fork":
        batch = _between(rng, 2, 64)
        return _fork(batch, rng.choice((0, 0, 1, 3, 9)), _between(rng, 4, max(8, 60000 // batch)), ragged, kv_heads, page, dtype, head)
    return _compact(_between(rng, 1, 48), _between(rng, 16, 3500), ragged, kv_heads, page, dtype, head)


def _lens(c):
    """Rows of each sequence: all alike, or spread unevenly between an eighth of the longest and the longest."""
    n, rows = c["batch"], c["rows"]
    if not c["ragged"]:
        return [rows] * n
    return [max(1, rows - (i * 37 % 101) * rows * 7 // 800) for i in range(n)]


# ------------------------------------------------------------------ inputs
class _Source:
    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dtype = dtype

    def normal(self, *shape, std=1.0):
        out = torch.empty(*shape, dtype=self.dtype, device="cuda")
        return out.normal_(0.0, std, generator=self.g)

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda").to(torch.int32)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pages(rows, page):
    return (rows + page - 1) // page


def _make_cache(s, c, lens, slots, width, n_pages, zeros=False):
    """A pool whose first sequences hold `lens` rows in pages scattered over it; what no sequence holds is stale."""
    G, d, page = c["kv_heads"], c["head"], c["page"]
    table = torch.full((slots, width), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    held = torch.zeros(slots, dtype=torch.int32, device="cuda")
    if lens:
        n = _i32(lens)
        held[: len(lens)] = n
        need = _pages(n, page)
        used = torch.arange(width, device="cuda") < need[:, None]
        order = s.order(n_pages)
        table[: len(lens)][used] = order[: sum(_pages(v, page) for v in lens)]
        refs[table[: len(lens)][used].long()] = 1
    if zeros:
        k, v = (torch.zeros(n_pages, page, G, d, dtype=s.dtype, device="cuda") for _ in range(2))
    else:
        # rows of a cache: normalised states times a weight matrix have about this spread
        k, v = (s.normal(n_pages, page, G, d, std=1.28) for _ in range(2))
    return dict(k=k, v=v, table=table, lens=held, refs=refs, page=page)


def _handle(cache):
    from paper_2505_24544_amd import binding as bx
    return bx.make_paged_cache(cache["k"], cache["v"], cache["table"], cache["lens"], cache["refs"])


def _desc(c, batch, queries, rows):
    from paper_2505_24544_amd import binding as bx
    return bx.make_desc(batch=batch, seq_q=queries, seq_kv=rows, hidden=128 * c.get("heads", c["kv_heads"]),
                        n_q_heads=c.get("heads", c["kv_heads"]), n_kv_heads=c["kv_heads"], head_dim=c["head"],
                        io_dtype=bx.BEAGLE_F32 if c["dtype"] == "f32" else bx.BEAGLE_BF16, flags=bx.BEAGLE_FLAG_ROPE)


def _workspace(desc, handle, which):
    from paper_2505_24544_amd import binding as bx
    n = bx.beagle_xattn_paged_workspace_bytes(desc, handle, getattr(bx, which))
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    c = case
    s = _Source(seed, torch.float32 if c["dtype"] == "f32" else torch.bfloat16)
    st = {"attend": _prepare_attend, "append": _prepare_append, "fork": _prepare_fork, "compact": _prepare_compact}[c["kind"]](c, s)
    st["case"] = dict(c)
    st["stream"] = torch.cuda.current_stream()
    return st


def _bits(s, *shape):
    """Random words of 32 bits, about one in four set."""
    a, b = (torch.randint(-(1 << 31), 1 << 31, shape, generator=s.g, device="cuda", dtype=torch.int64) for _ in range(2))
    return (a & b).to(torch.int32)


def _prepare_attend(c, s):
    B, M, H, T, page = c["batch"], c["queries"], c["heads"], c["drafted"], c["page"]
    true = _lens(c)
    lens = [n + T for n in true]
    width = _pages(max(lens), page)
    cache = _make_cache(s, c, lens, B, width, sum(_pages(n, page) for n in lens) + 8)
    words = _pages(T, 32)
    tree = _bits(s, B, M, words) if T else None
    st = dict(cache=cache, q=s.normal(B, M, H, c["head"], std=1.28), slots=torch.flip(torch.arange(B, dtype=torch.int32, device="cuda"), (0,)),
              n_true=_i32(true).flip(0).contiguous(), tree=tree, words=words, most=max(lens),
              o=torch.empty(B, M, H, c["head"], dtype=s.dtype, device="cuda"),
              lse=torch.empty(B, H, M, dtype=torch.float32, device="cuda"))
    if own:
        st["handle"] = _handle(cache)
        st["desc"] = _desc(c, B, M, st["most"])
        st["ws"] = _workspace(st["desc"], st["handle"], "BEAGLE_WS_PAGED_ATTEND")
    return st


def _prepare_append(c, s):
    B, n, G, d, page = c["batch"], c["states"], c["kv_heads"], c["head"], c["page"]
    lens = _lens(c)
    width = _pages(max(lens) + n, page)
    total = sum(_pages(v + n, page) for v in lens)
    cache = _make_cache(s, c, lens, B, width, total + total // 4 + 8)
    st = dict(cache=cache, slots=torch.flip(torch.arange(B, dtype=torch.int32, device="cuda"), (0,)),
              pos=_i32(lens).flip(0).contiguous(), k_new=s.normal(B, n, G, d, std=1.28), v_new=s.normal(B, n, G, d, std=1.28),
              short=torch.zeros(1, dtype=torch.int32, device="cuda"), shared=False)
    if own:
        st["handle"] = _handle(cache)
        st["desc"] = _desc(c, B, n, width * page)
        st["ws"] = _workspace(st["desc"], st["handle"], "BEAGLE_WS_PAGED_APPEND")
    return st


def _prepare_fork(c, s):
    """Slots 0 .. B-1 hold sequences, slots B .. 2B-1 are to take over rows of them, some of the same one."""
    B, n, G, d, page = c["batch"], c["states"], c["kv_heads"], c["head"], c["page"]
    lens = _lens(c)
    width = _pages(max(lens) + n, page)
    total = sum(_pages(v, page) for v in lens)
    cache = _make_cache(s, c, lens, 2 * B, width, total + total // 4 + B * (1 + _pages(n, page)) + 8)
    src = torch.randint(0, B, (B,), generator=s.g, device="cuda", dtype=torch.int32)
    # a branch leaves its parent at the parent's last row or a few rows before it
    back = torch.randint(0, 4, (B,), generator=s.g, device="cuda", dtype=torch.int32)
    rows = torch.clamp(cache["lens"][src.long()] - back, min=1).to(torch.int32)
    st = dict(cache=cache, src=src, rows=rows, dst=torch.arange(B, 2 * B, dtype=torch.int32, device="cuda"), slots=None,
              short=torch.zeros(1, dtype=torch.int32, device="cuda"), shared=True)
    if n:
        st.update(slots=st["dst"], pos=rows, k_new=s.normal(B, n, G, d, std=1.28), v_new=s.normal(B, n, G, d, std=1.28))
    if own:
        st["handle"] = _handle(cache)
        st["desc"] = _desc(c, B, max(n, 1), width * page)
        st["ws"] = _workspace(st["desc"], st["handle"], "BEAGLE_WS_PAGED_FORK")
        st["ws_append"] = _workspace(st["desc"], st["handle"], "BEAGLE_WS_PAGED_APPEND")
    return st


def _prepare_compact(c, s):
    lens, page = _lens(c), c["page"]
    width, live = _pages(max(lens), page), sum(_pages(n, page) for n in lens)
    cache = _make_cache(s, c, lens, c["batch"], width, 2 * live + 3)
    into = _make_cache(s, c, [], c["batch"], width, live + 5, zeros=True)
    st = dict(cache=cache, into=into, short=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if own:
        st["handle"], st["handle_into"] = _handle(cache), _handle(into)
        st["desc"] = _desc(c, c["batch"], 1, width * page)
        st["ws"] = _workspace(st["desc"], st["handle"], "BEAGLE_WS_PAGED_COMPACT")
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    return {"attend": _run_attend, "append": _run_append, "fork": _run_fork, "compact": _run_compact}[state["case"]["kind"]](state)


def _state_of(cache, st):
    return dict(k=cache["k"], v=cache["v"], table=cache["table"], lens=cache["lens"], refs=cache["refs"], short=st["short"])


def _run_attend(st):
    c = st["case"]
    if own:
        from paper_2505_24544_amd import binding as bx
        bx.beagle_xattn_paged_attend(st["desc"], st["handle"], st["q"], st["slots"], st["n_true"] if c["drafted"] else None, st["tree"],
                                     st["words"], c["window"], c["sinks"], st["o"], st["lse"], st["ws"], st["stream"])
        return dict(o=st["o"], lse=st["lse"])
    cache, q = st["cache"], st["q"]
    B, M, H, d = q.shape
    G, page, T = c["kv_heads"], c["page"], c["drafted"]
    slots = st["slots"].long()
    n = cache["lens"][slots].long()
    nt = st["n_true"].long() if T else n
    # the rows that some query may see: all of them, or the first ones and the window's
    if c["window"] and c["window"] + c["sinks"] < st["most"]:
        first = torch.arange(c["sinks"], device=q.device).expand(B, -1)
        last = (nt - c["window"])[:, None] + torch.arange(c["window"], device=q.device)
        j = torch.cat((first, last), 1)
        seen = (j >= 0) & (j < nt[:, None]) & ((torch.arange(j.shape[1], device=q.device) < c["sinks"]) | (j >= c["sinks"]))
        see = seen[:, None, :].expand(B, M, -1)
    else:
        j = torch.arange(st["most"], device=q.device).expand(B, -1)
        true = (j < nt[:, None]) & ((j < c["sinks"]) | (j >= nt[:, None] - c["window"])) if c["window"] else j < nt[:, None]
        seen, see = j < n[:, None], true[:, None, :].expand(B, M, -1)
        if T:
            t = j - nt[:, None]
            inside = (t >= 0) & (t < T)
            t = t.clamp(0, T - 1)
            word = torch.gather(st["tree"], 2, (t // 32)[:, None, :].expand(B, M, -1))
            see = see | (inside[:, None, :] & ((word >> (t % 32)[:, None, :]) & 1).bool())
    j = torch.where(seen, j, 0)
    at = (cache["table"][slots].long().gather(1, j // page) * page + j % page).clamp(min=0)
    k = cache["k"].view(-1, G, d)[at].float()
    v = cache["v"].view(-1, G, d)[at].float()
    qf = q.float().view(B, M, G, H // G, d).permute(0, 2, 1, 3, 4).reshape(B, G, M * (H // G), d)
    x = torch.matmul(qf, k.permute(0, 2, 3, 1)).view(B, G, M, H // G, -1) / math.sqrt(d)
    x = x.masked_fill(~see[:, None, :, None, :], float("-inf"))
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isneginf(top), 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, G, M * (H // G), -1), v.permute(0, 2, 1, 3)).view(B, G, M, H // G, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(B, M, H, d).to(q.dtype)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 1, 3, 2).reshape(B, H, M)
    return dict(o=o, lse=lse)


def _append_plain(st):
    """Trims every slot to its first pos rows, takes the lowest free pages, copies shared pages and writes the rows."""
    cache, slots, pos = st["cache"], st["slots"].long(), st["pos"].long()
    k_new, v_new, page = st["k_new"], st["v_new"], cache["page"]
    B, n, G, d = k_new.shape
    table, refs = cache["table"], cache["refs"]
    W, P = table.shape[1], refs.shape[0]
    mine = table[slots].long()
    col = torch.arange(W, device=pos.device).expand(B, -1)
    old, keep, want = _pages(cache["lens"][slots].long(), page)[:, None], _pages(pos, page)[:, None], _pages(pos + n, page)[:, None]
    # released pages; a page of the pool counts one for each of them
    gone = (col >= keep) & (col < old)
    refs.index_add_(0, torch.where(gone, mine, 0).reshape(-1), -gone.reshape(-1).to(torch.int32))
    last = mine.gather(1, (pos // page).clamp(max=W - 1)[:, None]).squeeze(1)      # the page of row pos, where it is partly kept
    part = pos % page != 0
    copied = part & (refs[torch.where(part, last, 0)] > 1)
    new = ((col >= keep) & (col < want)) | (copied[:, None] & (col == (pos // page)[:, None]))
    # the lowest free pages in order, entry after entry (the pool has them)
    st["short"].copy_((new.sum() - (refs == 0).sum()).clamp(min=0))
    order = torch.argsort((refs != 0).to(torch.int8), stable=True)
    rank = torch.cumsum(new.reshape(-1), 0).view(B, W) - 1
    taken = order[rank.clamp(0, P - 1)]
    mine = torch.where(new, taken, mine)
    refs.index_add_(0, torch.where(copied, last, 0), -copied.to(torch.int32))
    refs.index_add_(0, torch.where(new, taken, 0).reshape(-1), new.reshape(-1).to(torch.int32))
    table[slots] = mine.to(torch.int32)
    cache["lens"][slots] = (pos + n).to(torch.int32)
    # rows: K rotated at its position
    row = pos[:, None] + torch.arange(n, device=pos.device)
    angle = row.double()[:, :, None] * ROPE_BASE ** (-2.0 * torch.arange(d // 2, device=pos.device, dtype=torch.float64) / d)
    cos, sin = angle.cos().float()[:, :, None, :], angle.sin().float()[:, :, None, :]
    a, b = k_new.float().split(d // 2, dim=-1)
    k_rot = torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(k_new.dtype)
    if st["shared"]:
        fresh = torch.where(copied, mine.gather(1, (pos // page).clamp(max=W - 1)[:, None]).squeeze(1), 0)
        src = torch.where(copied, last, 0)
        kept = (torch.arange(page, device=pos.device) < (pos % page)[:, None])[:, :, None, None] & copied[:, None, None, None]
        # entries that copy nothing put page 0 back as it is, behind those that write it
        turn = torch.argsort(copied.to(torch.int8), stable=True)
        for name in ("k", "v"):
            pages = torch.where(kept, cache[name][src], cache[name][fresh])
            cache[name][fresh[turn]] = pages[turn]
    at = mine.gather(1, (row // page).clamp(max=W - 1)) * page + row % page
    k, v = (cache[name].view(-1, G, d) for name in ("k", "v"))
    k[at.reshape(-1)] = k_rot.view(-1, G, d)
    v[at.reshape(-1)] = v_new.reshape(-1, G, d)


def _append_own(st, ws):
    from paper_2505_24544_amd import binding as bx
    bx.beagle_xattn_paged_append(st["desc"], st["handle"], st["slots"], st["pos"], None, st["k_new"], st["v_new"], st["short"], ws,
                                 st["stream"])


def _run_append(st):
    if own:
        _append_own(st, st["ws"])
    else:
        _append_plain(st)
    return _state_of(st["cache"], st)


def _run_fork(st):
    cache = st["cache"]
    if own:
        from paper_2505_24544_amd import binding as bx
        bx.beagle_xattn_paged_fork(st["desc"], st["handle"], st["dst"], st["src"], st["rows"], st["ws"], st["stream"])
        if st["slots"] is not None:
            _append_own(st, st["ws_append"])
        return _state_of(cache, st)
    table, refs, lens, page = cache["table"], cache["refs"], cache["lens"], cache["page"]
    dst, src = st["dst"].long(), st["src"].long()
    col = torch.arange(table.shape[1], device=dst.device)
    rows = torch.minimum(st["rows"], lens[src]).clamp(min=0)
    before, after = table[dst].long(), table[src]
    gone = col < _pages(lens[dst], page)[:, None]
    held = col < _pages(rows, page)[:, None]
    refs.index_add_(0, torch.where(gone, before, 0).reshape(-1), -gone.reshape(-1).to(torch.int32))
    refs.index_add_(0, torch.where(held, after.long(), 0).reshape(-1), held.reshape(-1).to(torch.int32))
    table[dst] = torch.where(held, after, -1)
    lens[dst] = rows
    if st["slots"] is not None:
        _append_plain(st)
    return _state_of(cache, st)


def _run_compact(st):
    cache, into = st["cache"], st["into"]
    if own:
        from paper_2505_24544_amd import binding as bx
        bx.beagle_xattn_paged_compact(st["desc"], st["handle"], st["handle_into"], st["short"], st["ws"], st["stream"])
        return _state_of(into, st)
    live = cache["refs"] > 0
    count = live.sum()
    P = into["refs"].shape[0]
    order = torch.argsort((~live).to(torch.int8), stable=True)[:P]       # the live pages in order of their number
    moved = torch.arange(P, device=order.device) < count
    number = torch.cumsum(live, 0) - 1
    held = torch.arange(cache["table"].shape[1], device=order.device) < _pages(cache["lens"], cache["page"])[:, None]
    mine = cache["table"].long().clamp(min=0)
    into["table"].copy_(torch.where(held, number[mine], -1))
    into["lens"].copy_(cache["lens"])
    into["refs"].copy_(torch.where(moved, cache["refs"][order], 0))
    st["short"].copy_((count - P).clamp(min=0))
    for name in ("k", "v"):
        into[name].copy_(torch.where(moved[:, None, None, None], cache[name][order], into[name]))
    return _state_of(into, st)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    e, d, G, page, lens = (4 if c["dtype"] == "f32" else 2), c["head"], c["kv_heads"], c["page"], _lens(c)
    row = 2 * G * d * e                                              # K and V
    if c["kind"] == "attend":
        B, M, H = c["batch"], c["queries"], c["heads"]
        seen = sum(min(n, c["window"] + c["sinks"]) if c["window"] else n for n in lens) + B * c["drafted"]
        return dict(bytes=seen * row + 2 * B * M * H * d * e + 4 * B * M * H + 4 * seen // page + 4 * B * M * _pages(c["drafted"], 32),
                    flops=4 * d * H * M * seen)
    if c["kind"] == "compact":
        live = sum(_pages(n, page) for n in lens)
        return dict(bytes=2 * sum(lens) * row + 16 * live, flops=0)
    n = c["states"]
    moved, flops = 2 * c["batch"] * n * row, 3 * c["batch"] * n * G * d
    if c["kind"] == "append":
        return dict(bytes=moved + 8 * c["batch"] * _pages(n, page), flops=flops)
    # a branch copies half a page on average
    moved += 2 * c["batch"] * (page // 2) * row if n else 0
    return dict(bytes=moved + 16 * sum(_pages(v, page) for v in lens), flops=flops)


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["kind"] == "attend":
        return _exact_attend(c, st)
    if c["kind"] == "append" or (c["kind"] == "fork" and c["states"]):
        cache = st["cache"]
        _follow(c, st)
        # the only numbers that are computed: the rotated K rows; where they go is followed step by step on the host
        return dict(k=_exact_rows(c, st, cache), v=None, table=None, lens=None, refs=None, short=None)
    return None


def _exact_attend(c, st):
    """Sequence after sequence, query after query: a softmax over the rows that the definition names."""
    B, M, H, d = st["q"].shape
    G, page, T = c["kv_heads"], c["page"], c["drafted"]
    cache = st["cache"]
    o = torch.zeros(B, M, H, d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, M), float("-inf"), dtype=torch.float64, device="cuda")
    slots, true = st["slots"].tolist(), st["n_true"].tolist()
    for b in range(B):
        n = int(cache["lens"][slots[b]])
        nt = true[b] if T else n
        for m in range(M):
            if c["window"]:
                ids = sorted(set(range(min(c["sinks"], nt))) | set(range(max(0, nt - c["window"]), nt)))
            else:
                ids = list(range(nt))
            words = st["tree"][b, m].tolist() if T else []
            ids += [nt + t for t in range(T) if (words[t // 32] >> (t % 32)) & 1]
            if not ids:
                continue
            if m == 0 or T:
                j = torch.tensor(ids, device="cuda")
                page_of = cache["table"][slots[b]][torch.div(j, page, rounding_mode="floor")].long()
                k = cache["k"][page_of, j % page].double().transpose(0, 1)
                v = cache["v"][page_of, j % page].double().transpose(0, 1)
            q = st["q"][b, m].double().view(G, H // G, d)
            x = torch.bmm(q, k.transpose(1, 2).contiguous()) * d ** -0.5
            z = torch.logsumexp(x, -1, keepdim=True)
            o[b, m] = torch.bmm(torch.exp(x - z), v).reshape(H, d)
            lse[b, :, m] = z.reshape(H)
    return dict(o=o, lse=lse)


def _follow(c, st):
    """Bookkeeping of fork and append on lists: which page each entry's rows go to, and which pages are copied."""
    cache, page = st["cache"], c["page"]
    table, lens, refs = cache["table"].tolist(), cache["lens"].tolist(), cache["refs"].tolist()
    if c["kind"] == "fork":
        old = [list(r) for r in table]
        had = list(lens)
        for a, b, n in zip(st["dst"].tolist(), st["src"].tolist(), st["rows"].tolist()):
            for p in old[a][: _pages(had[a], page)]:
                refs[p] -= 1
            table[a] = old[b][: _pages(n, page)] + [-1] * (len(old[b]) - _pages(n, page))
            for p in table[a][: _pages(n, page)]:
                refs[p] += 1
            lens[a] = n
    st["moves"], st["targets"] = [], []
    n = c["states"]
    todo = list(zip(st["slots"].tolist(), st["pos"].tolist()))
    for a, pos in todo:
        for p in table[a][_pages(pos, page): _pages(lens[a], page)]:
            refs[p] -= 1
    shared = [pos % page != 0 and refs[table[a][pos // page]] > 1 for a, pos in todo]
    free = [p for p, r in enumerate(refs) if r == 0]
    for (a, pos), cow in zip(todo, shared):
        if cow:
            p = free.pop(0)
            st["moves"].append((table[a][pos // page], p, pos % page))
            table[a][pos // page] = p
        for i in range(_pages(pos, page), _pages(pos + n, page)):
            table[a][i] = free.pop(0)
        st["targets"].append([table[a][r // page] * page + r % page for r in range(pos, pos + n)])


def _exact_rows(c, st, cache):
    k = cache["k"].double()
    page, d = c["page"], c["head"]
    for src, dst, rows in st["moves"]:
        k[dst, :rows] = k[src, :rows]
    at = torch.tensor(st["targets"], device="cuda")
    x = st["k_new"].double()
    turn = (st["pos"].double()[:, None] + torch.arange(c["states"], device="cuda", dtype=torch.float64))[:, :, None]
    turn = turn * torch.exp(-2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d * math.log(ROPE_BASE))
    z = torch.polar(torch.ones_like(turn), turn)[:, :, None, :] * torch.complex(x[..., : d // 2].contiguous(), x[..., d // 2:].contiguous())
    k.view(-1, *k.shape[2:])[at.reshape(-1)] = torch.cat((z.real, z.imag), -1).view(-1, *k.shape[2:])
    return k
