"""Attention over long and over shared contexts in the paged cache, as cases that can be timed and checked.

Sequences that branched from one another share the rows of their common prefix: `shared` attends to a prefix once for all
entries of a group, and to every entry's own rows behind it.  Of a long context a query needs a few pages: `bounds` keeps, for
every page and head, the least and the greatest value of each channel of its keys, `select` takes from them the pages whose keys
can give the largest scores, and `blocks` attends to the rows of those pages, of the first rows and of the last ones.

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


# ------------------------------------------------------------------ the cases
def _shared(batch, groups, queries, prefix, suffix, drafted, heads, kv_heads, page, dtype="bf16", head=128, name=None):
    c = dict(kind="shared", batch=batch, groups=groups, queries=queries, prefix=prefix, suffix=suffix, drafted=drafted, heads=heads,
             kv_heads=kv_heads, page=page, dtype=dtype, head=head)
    return dict(c, name=name) if name else c


def _bounds(batch, rows, new, kv_heads, page, dtype="bf16", head=128, name=None):
    c = dict(kind="bounds", batch=batch, rows=rows, new=new, heads=kv_heads, kv_heads=kv_heads, page=page, dtype=dtype, head=head)
    return dict(c, name=name) if name else c


def _select(batch, queries, rows, pages, window, sinks, heads, kv_heads, page, drafted=0, dtype="bf16", head=128, name=None):
    c = dict(kind="select", batch=batch, queries=queries, rows=rows, pages=pages, window=window, sinks=sinks, heads=heads,
             kv_heads=kv_heads, page=page, drafted=drafted, dtype=dtype, head=head)
    return dict(c, name=name) if name else c


def _blocks(*args, **kw):
    return dict(_select(*args, **kw), kind="blocks")


def listed():
    return [
        # a few branches of a short sequence, the fp32 relative of the reference problem: all launch latency
        _shared(4, 1, 2, 300, 40, 0, 4, 2, 8, dtype="f32", head=64, name="shared_branches_f32"),
        # many users under one system prompt, grouped queries, one query each
        _shared(32, 1, 1, 4000, 700, 0, 32, 8, 16, name="shared_prompt_8b"),
        # three documents that four users each draft trees on, at the 13B shape
        _shared(12, 3, 10, 6000, 500, 50, 40, 40, 32, name="shared_tree_13b"),
        # a wide beam over one long document, several queries each
        _shared(64, 1, 4, 16000, 300, 0, 32, 8, 64, name="shared_beam_8b"),
        # after the accepted tokens of one iteration entered the caches of a batch
        _bounds(64, 4000, 5, 8, 16, name="bounds_accepted"),
        # after prompts entered the cache
        _bounds(6, 8000, 8000, 32, 64, name="bounds_prompts"),
        # one user's draft query over a document
        _select(1, 1, 6000, 32, 256, 4, 32, 32, 32, name="select_one"),
        # a batch of long chats with grouped queries
        _select(32, 4, 20000, 40, 512, 4, 32, 8, 64, name="select_batch_8b"),
        # the paper's tree on long contexts at the 13B shape
        _select(4, 10, 32768, 100, 512, 4, 40, 40, 32, drafted=50, name="select_tree_13b"),
        # the same three steps on: the attention over what was selected
        _blocks(6, 2, 1500, 20, 100, 5, 4, 2, 8, dtype="f32", head=64, name="blocks_f32"),
        _blocks(32, 4, 20000, 40, 512, 4, 32, 8, 64, name="blocks_batch_8b"),
        _blocks(4, 10, 32768, 100, 512, 4, 40, 40, 32, drafted=50, name="blocks_tree_13b"),
    ]


def _between(rng, lo, hi):
    """A whole number in [lo, hi], evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("shared", "shared", "shared", "bounds", "select", "select", "blocks", "blocks"))
    f32 = rng.random() < 0.25
    heads, kv_heads, head = rng.choice(HEADS_F32) if f32 else rng.choice(HEADS) + (128,)
    dtype, page = "f32" if f32 else "bf16", rng.choice((8, 16, 16, 32, 64, 128))
    queries = rng.choice((1, 1, 1, 2, 4, 7, 10, 16))
    drafted = rng.choice((0, 0, rng.randint(1, 60))) if queries > 1 else 0
    batch = _between(rng, 1, 64)
    if kind == "shared":
        batch = max(batch, 2)
        groups = _between(rng, 1, max(1, min(8, batch // 2)))
        # no more scores in all than the largest listed case has
        most = (1 << 19 if f32 else 1 << 27) // (batch * queries * heads)
        prefix = _between(rng, 1, max(2, min(16000, most, (20000 if f32 else 640000 // kv_heads) // groups)))
        suffix = _between(rng, 1, max(2, min(1000, (4000 if f32 else 640000 // kv_heads) // batch)))
        return _shared(batch, groups, queries, prefix, suffix, drafted, heads, kv_heads, page, dtype, head)
    # no more rows in all than the largest listed cases have
    most = (20000 if f32 else 81920 * 40 // kv_heads) // batch
    if kind == "bounds":
        rows = _between(rng, 2 * page, max(2 * page + 1, min(32768, most if f32 else most // 3)))
        return _bounds(batch, rows, rng.choice((rows, _between(rng, 1, rows))), kv_heads, page, dtype, head)
    rows = _between(rng, 4 * page, max(4 * page + 1, min(32768, most)))
    args = (batch, queries, rows, _between(rng, 1, max(1, min(128, 4096 // page, rows // page))), rng.choice((0, _between(rng, 1, min(1024, rows // 2)))),
            rng.choice((0, 1, 4, 4, 16, 100)), heads, kv_heads, page)
    return (_select if kind == "select" else _blocks)(*args, drafted=drafted, dtype=dtype, head=head)


def _spread(n, most):
    """n lengths, spread unevenly between an eighth of the longest and the longest."""
    return [max(1, most - (i * 37 % 101) * most * 7 // 800) for i in range(n)]


def _group_first(c):
    """First entry of every group, and the end: groups of unequal sizes, none empty."""
    n, g = c["batch"], c["groups"]
    spare, sizes = n - g, [1] * g
    for i in range(g):
        take = spare if i == g - 1 else min(spare, max(0, (n // g - 1) + (i % 3 - 1) * (n // (4 * g))))
        sizes[i] += take
        spare -= take
    first = [0]
    for s in sizes:
        first.append(first[-1] + s)
    return first


def _prefixes(c):
    return _spread(c["groups"], c["prefix"])


def _candidates(c, true):
    """First and one past the last of the pages that are not seen anyway."""
    sp = -(-c["sinks"] // c["page"])
    return sp, max(sp, max(true - c["window"], 0) // c["page"])


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


def _pool(s, c, n_pages):
    # rows of a cache: normalised states times a weight matrix have about this spread
    return [s.normal(n_pages, c["page"], c["kv_heads"], c["head"], std=1.28) for _ in range(2)]


def _make_cache(s, c, lens):
    """A pool in which slot i holds lens[i] rows in pages scattered over it; what no sequence holds is stale."""
    page = c["page"]
    need = [_pages(n, page) for n in lens]
    n_pages = sum(need) + 8
    order = s.order(n_pages)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(max(need), device="cuda") < _i32(need)[:, None]] = order[: sum(need)]
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[order[: sum(need)].long()] = 1
    k, v = _pool(s, c, n_pages)
    return dict(k=k, v=v, table=table, lens=_i32(lens), refs=refs, page=page)


def _make_branches(s, c, slots, first, shared, own_rows):
    """A pool in which the entries of a group share the whole pages of their prefix; the page that the prefix ends in is
    each one's own, as it is after they have appended to it."""
    page, B = c["page"], c["batch"]
    group = [g for g in range(c["groups"]) for _ in range(first[g], first[g + 1])]
    lens = [shared[group[b]] + own_rows[b] for b in range(B)]
    whole = [n // page for n in shared]
    need = [_pages(lens[b], page) - whole[group[b]] for b in range(B)]
    n_pages = sum(whole) + sum(need) + 8
    order = s.order(n_pages).tolist()
    prefix = [[order.pop() for _ in range(n)] for n in whole]
    width = max(_pages(n, page) for n in lens)
    table, refs, held, ends = [[-1] * width for _ in range(B)], [0] * n_pages, [0] * B, [[], []]
    for b in range(B):
        row = prefix[group[b]] + [order.pop() for _ in range(need[b])]
        table[slots[b]][: len(row)] = row
        held[slots[b]] = lens[b]
        for p in row:
            refs[p] += 1
        lead = first[group[b]]
        if b != lead and shared[group[b]] % page:
            ends[0].append((table[slots[lead]][whole[group[b]]], shared[group[b]] % page))
            ends[1].append(row[whole[group[b]]])
    k, v = _pool(s, c, n_pages)
    if ends[0]:
        src, dst = _i32([e[0] for e in ends[0]]).long(), _i32(ends[1]).long()
        kept = (torch.arange(page, device="cuda") < _i32([e[1] for e in ends[0]])[:, None])[:, :, None, None]
        for x in (k, v):
            x[dst] = torch.where(kept, x[src], x[dst])
    return dict(k=k, v=v, table=_i32(table), lens=_i32(held), refs=_i32(refs), page=page)


def _handle(cache):
    from paper_2505_24544_amd import binding as bx
    return bx.make_paged_cache(cache["k"], cache["v"], cache["table"], cache["lens"], cache["refs"])


def _desc(c, rows):
    from paper_2505_24544_amd import binding as bx
    return bx.make_desc(batch=c["batch"], seq_q=c.get("queries", 1), seq_kv=rows, hidden=128 * c["heads"], n_q_heads=c["heads"],
                        n_kv_heads=c["kv_heads"], head_dim=c["head"], io_dtype=bx.BEAGLE_F32 if c["dtype"] == "f32" else bx.BEAGLE_BF16)


def _workspace(desc, handle, which):
    from paper_2505_24544_amd import binding as bx
    n = bx.beagle_xattn_paged_workspace_bytes(desc, handle, getattr(bx, which))
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    c = case
    s = _Source(seed, torch.float32 if c["dtype"] == "f32" else torch.bfloat16)
    st = {"shared": _prepare_shared, "bounds": _prepare_bounds, "select": _prepare_pages, "blocks": _prepare_pages}[c["kind"]](c, s)
    st["case"] = dict(c)
    st["stream"] = torch.cuda.current_stream()
    return st


def _bits(s, *shape):
    """Random words of 32 bits, about one in four set."""
    a, b = (torch.randint(-(1 << 31), 1 << 31, shape, generator=s.g, device="cuda", dtype=torch.int64) for _ in range(2))
    return (a & b).to(torch.int32)


def _queries(s, c):
    B, M, H, d, T = c["batch"], c["queries"], c["heads"], c["head"], c["drafted"]
    words = _pages(T, 32)
    return dict(q=s.normal(B, M, H, d, std=1.28), tree=_bits(s, B, M, words) if T else None, words=words,
                o=torch.empty(B, M, H, d, dtype=s.dtype, device="cuda"), lse=torch.empty(B, H, M, dtype=torch.float32, device="cuda"))


def _prepare_shared(c, s):
    B, T = c["batch"], c["drafted"]
    first, shared = _group_first(c), _prefixes(c)
    group = [g for g in range(c["groups"]) for _ in range(first[g], first[g + 1])]
    mine = _spread(B, c["suffix"])
    slots = list(range(B - 1, -1, -1))
    true = [shared[group[b]] + mine[b] for b in range(B)]
    cache = _make_branches(s, c, slots, first, shared, [n + T for n in mine])
    st = dict(cache=cache, slots=_i32(slots), first=first, shared=shared, true=true, group_first=_i32(first), n_shared=_i32(shared),
              n_true=_i32(true) if T else None, most=max(true) + T, **_queries(s, c))
    if own:
        st["handle"] = _handle(cache)
        st["desc"] = _desc(c, st["most"])
        st["ws"] = _workspace(st["desc"], st["handle"], "BEAGLE_WS_PAGED_SHARED")
    return st


def _prepare_bounds(c, s):
    lens = _spread(c["batch"], c["rows"])
    cache = _make_cache(s, c, lens)
    st = dict(cache=cache, slots=torch.flip(torch.arange(c["batch"], dtype=torch.int32, device="cuda"), (0,)),
              first=_i32([max(n - c["new"], 0) for n in lens]).flip(0).contiguous(),
              bounds=torch.zeros(cache["k"].shape[0], c["kv_heads"], 2, c["head"], dtype=s.dtype, device="cuda"), most=max(lens))
    if own:
        st["handle"] = _handle(cache)
        st["desc"] = _desc(c, st["most"])
    return st


def _prepare_pages(c, s):
    B, T, page = c["batch"], c["drafted"], c["page"]
    true = _spread(B, c["rows"])
    cache = _make_cache(s, c, [n + T for n in true])
    st = dict(cache=cache, slots=torch.flip(torch.arange(B, dtype=torch.int32, device="cuda"), (0,)), true=true[::-1],
              n_true=_i32(true[::-1]) if T else None, most=max(true) + T, **_queries(s, c))
    G, n = c["kv_heads"], c["pages"]
    if c["kind"] == "select":
        st["bounds"] = torch.stack((cache["k"].amin(1), cache["k"].amax(1)), 2).contiguous()
        st["pages"] = torch.empty(B, G, n, dtype=torch.int32, device="cuda")
    else:
        # some selection of the candidates for every entry and head
        spans = [_candidates(c, t) for t in st["true"]]
        lo, hi = (_i32([x[i] for x in spans])[:, None, None] for i in range(2))
        width = max(max(x[1] for x in spans), n)
        col = torch.arange(width, device="cuda")
        luck = torch.rand(B, G, width, generator=s.g, device="cuda")
        luck = torch.where((col >= lo) & (col < hi), luck, 2.0)
        order = torch.argsort(luck, -1)[..., :n]
        order = torch.where(torch.gather(luck, 2, order) < 2.0, order, 1 << 30)
        order = torch.sort(order, -1).values
        st["pages"] = torch.where(order < 1 << 30, order, -1).to(torch.int32).contiguous()
    if own:
        st["handle"] = _handle(cache)
        st["desc"] = _desc(c, st["most"])
        st["ws"] = _workspace(st["desc"], st["handle"], "BEAGLE_WS_PAGED_SELECT" if c["kind"] == "select" else "BEAGLE_WS_PAGED_BLOCKS")
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    return {"shared": _run_shared, "bounds": _run_bounds, "select": _run_select, "blocks": _run_blocks}[state["case"]["kind"]](state)


def _tree_bits(st, T):
    """Drafted row t as the queries of each entry see it: [B, M, T]."""
    t = torch.arange(T, device="cuda")
    return ((st["tree"][:, :, t // 32] >> (t % 32)) & 1).bool()


def _over(total, o, top):
    """Sums of a softmax -> its result and the log-sum-exp."""
    return torch.where(total > 0, o / total, 0.0), (top + torch.log(total)).squeeze(-1)


def _finite_top(*scores):
    top = torch.stack([x.amax(-1, keepdim=True) for x in scores]).amax(0)
    return torch.where(torch.isneginf(top), 0.0, top)


def _run_shared(st):
    c = st["case"]
    if own:
        from paper_2505_24544_amd import binding as bx
        bx.beagle_xattn_paged_attend_shared(st["desc"], st["handle"], st["q"], st["slots"], st["group_first"], st["n_shared"], c["groups"],
                                            st["n_true"], st["tree"], st["words"], st["o"], st["lse"], st["ws"], st["stream"])
        return dict(o=st["o"], lse=st["lse"])
    cache, q = st["cache"], st["q"]
    B, M, H, d = q.shape
    G, page, T = c["kv_heads"], c["page"], c["drafted"]
    rep = H // G
    slots, table = st["slots"].long(), cache["table"]
    k_rows, v_rows = cache["k"].view(-1, G, d), cache["v"].view(-1, G, d)
    qf = q.float().view(B, M, G, rep, d).permute(0, 2, 1, 3, 4).reshape(B, G, M * rep, d) / math.sqrt(d)
    o = torch.empty(B, G, M * rep, d, device=q.device)
    lse = torch.empty(B, G, M * rep, device=q.device)
    tree = _tree_bits(st, T) if T else None
    for g, n in enumerate(st["shared"]):
        lo, hi = st["first"][g], st["first"][g + 1]
        E, mine = hi - lo, slots[lo:hi]
        # the prefix, once for all entries of the group
        j = torch.arange(n, device=q.device)
        at = table[mine[0]].long()[j // page] * page + j % page
        kp, vp = k_rows[at].float().permute(1, 2, 0), v_rows[at].float().transpose(0, 1)
        qg = qf[lo:hi].transpose(0, 1).reshape(G, E * M * rep, d)
        xp = torch.matmul(qg, kp)
        # the rows of each
        have = cache["lens"][mine].long()
        true = st["n_true"][lo:hi].long() if T else have
        j = n + torch.arange(max(st["true"][lo:hi]) + T - n, device=q.device)
        held = j < have[:, None]
        at = torch.where(held, torch.gather(table[mine].long(), 1, (j // page).expand(E, -1)) * page + j % page, 0).clamp(min=0)
        ks, vs = k_rows[at].float().permute(0, 2, 3, 1), v_rows[at].float().permute(0, 2, 1, 3)
        xs = torch.matmul(qf[lo:hi], ks).view(E, G, M, rep, -1)
        see = (j < true[:, None])[:, None, :].expand(E, M, -1)
        if T:
            t = j - true[:, None]
            drafted = torch.gather(tree[lo:hi], 2, t.clamp(0, T - 1)[:, None, :].expand(E, M, -1))
            see = see | (((t >= 0) & (t < T))[:, None, :] & drafted)
        xs = xs.masked_fill(~see[:, None, :, None, :], float("-inf")).view(E, G, M * rep, -1)
        top = _finite_top(xp.view(G, E, M * rep, n).transpose(0, 1), xs)
        pp = torch.exp(xp - top.transpose(0, 1).reshape(G, E * M * rep, 1))
        ps = torch.exp(xs - top)
        total = pp.sum(-1).view(G, E, M * rep, 1).transpose(0, 1) + ps.sum(-1, keepdim=True)
        sums = torch.matmul(pp, vp).view(G, E, M * rep, d).transpose(0, 1) + torch.matmul(ps, vs)
        o[lo:hi], lse[lo:hi] = _over(total, sums, top)
    o = o.view(B, G, M, rep, d).permute(0, 2, 1, 3, 4).reshape(B, M, H, d).to(q.dtype)
    return dict(o=o, lse=lse.view(B, G, M, rep).permute(0, 1, 3, 2).reshape(B, H, M))


def _run_bounds(st):
    cache, bounds = st["cache"], st["bounds"]
    if own:
        from paper_2505_24544_amd import binding as bx
        bx.beagle_xattn_paged_bounds(st["desc"], st["handle"], st["slots"], st["first"], bounds, st["stream"])
        return bounds
    page, slots = cache["page"], st["slots"].long()
    # whole pages that hold a row from `first` on
    col = torch.arange(cache["table"].shape[1], device=slots.device)
    whole = (col >= torch.div(st["first"], page, rounding_mode="floor")[:, None]) & ((col + 1) * page <= cache["lens"][slots][:, None])
    at = cache["table"][slots][whole].long()
    k = cache["k"][at]
    bounds[at] = torch.stack((k.amin(1), k.amax(1)), 2)
    return bounds


def _run_select(st):
    c = st["case"]
    if own:
        from paper_2505_24544_amd import binding as bx
        bx.beagle_xattn_paged_select(st["desc"], st["handle"], st["q"], st["slots"], st["n_true"], st["bounds"], c["window"], c["sinks"],
                                     c["pages"], st["pages"], st["ws"], st["stream"])
        return st["pages"]
    cache, q, n = st["cache"], st["q"], c["pages"]
    B, M, H, d = q.shape
    G, page = c["kv_heads"], c["page"]
    slots = st["slots"].long()
    true = (st["n_true"] if st["n_true"] is not None else cache["lens"][slots]).long()
    sp = _pages(c["sinks"], page)
    wp = torch.clamp(torch.div((true - c["window"]).clamp(min=0), page, rounding_mode="floor"), min=sp)
    col = torch.arange(cache["table"].shape[1], device=q.device)
    there = (col >= sp) & (col < wp[:, None])
    table = torch.where(there, cache["table"][slots], 0).long()
    # the greatest score that a key between the bounds can have; what ranks pages is added up in 64 bits
    qf = q.double().view(B, M, G, H // G, d).permute(0, 2, 1, 3, 4).reshape(B, G, -1, d)
    score = torch.empty(B, G, len(col), device=q.device)
    for b in range(B):
        lo, hi = st["bounds"][table[b]].double().permute(2, 1, 3, 0)          # [G, d, pages] each
        x = torch.matmul(qf[b].clamp(min=0), hi) + torch.matmul(qf[b].clamp(max=0), lo)
        score[b] = x.amax(1).float()
    score = score.masked_fill(~there[:, None, :], float("-inf"))
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :n]
    picked = torch.gather(there[:, None, :].expand(B, G, -1), 2, order)
    order = torch.sort(torch.where(picked, order, 1 << 30), -1).values
    st["pages"].fill_(-1)
    st["pages"][..., : order.shape[-1]] = torch.where(order < 1 << 30, order, -1).to(torch.int32)
    return st["pages"]


def _run_blocks(st):
    c = st["case"]
    if own:
        from paper_2505_24544_amd import binding as bx
        bx.beagle_xattn_paged_attend_blocks(st["desc"], st["handle"], st["q"], st["slots"], st["n_true"], st["tree"], st["words"],
                                            c["window"], c["sinks"], st["pages"], c["pages"], st["o"], st["lse"], st["ws"], st["stream"])
        return dict(o=st["o"], lse=st["lse"])
    cache, q = st["cache"], st["q"]
    B, M, H, d = q.shape
    G, page, T, N = c["kv_heads"], c["page"], c["drafted"], c["pages"]
    rep = H // G
    slots = st["slots"].long()
    have = cache["lens"][slots].long()
    true = st["n_true"].long() if T else have
    sp = _pages(c["sinks"], page)
    wp = torch.clamp(torch.div((true - c["window"]).clamp(min=0), page, rounding_mode="floor"), min=sp)
    # the pages that a kv head sees: the first ones, the listed ones, the last ones
    tail = torch.arange(_pages(c["window"] + T, page) + 1, device=q.device)
    cols = torch.cat((torch.arange(sp, device=q.device).expand(B, G, sp), st["pages"].long(),
                      (wp[:, None] + tail)[:, None, :].expand(B, G, -1)), 2)
    cols = torch.where((cols >= 0) & (cols * page < have[:, None, None]), cols, -1)
    j = (cols[..., None] * page + torch.arange(page, device=q.device)).view(B, G, -1)
    there = (cols[..., None] >= 0).expand(*cols.shape, page).reshape(B, G, -1) & (j < have[:, None, None])
    numbers = torch.gather(cache["table"][slots].long()[:, None, :].expand(B, G, -1), 2, cols.clamp(min=0))
    at = (numbers.clamp(min=0)[..., None] * page + torch.arange(page, device=q.device)).view(B, G, -1)
    head = torch.arange(G, device=q.device)[None, :, None]
    k, v = (cache[name].view(-1, G, d)[at, head].float() for name in ("k", "v"))
    qf = q.float().view(B, M, G, rep, d).permute(0, 2, 1, 3, 4).reshape(B, G, M * rep, d) / math.sqrt(d)
    x = torch.matmul(qf, k.transpose(2, 3)).view(B, G, M, rep, -1)
    see = (there & (j < true[:, None, None]))[:, :, None, :].expand(B, G, M, -1)
    if T:
        t = j - true[:, None, None]
        drafted = torch.gather(_tree_bits(st, T)[:, None].expand(B, G, M, T), 3, t.clamp(0, T - 1)[:, :, None, :].expand(B, G, M, -1))
        see = see | ((there & (t >= 0) & (t < T))[:, :, None, :] & drafted)
    x = x.masked_fill(~see[:, :, :, None, :], float("-inf")).view(B, G, M * rep, -1)
    top = _finite_top(x)
    p = torch.exp(x - top)
    o, lse = _over(p.sum(-1, keepdim=True), torch.matmul(p, v), top)
    o = o.view(B, G, M, rep, d).permute(0, 2, 1, 3, 4).reshape(B, M, H, d).to(q.dtype)
    return dict(o=o, lse=lse.view(B, G, M, rep).permute(0, 1, 3, 2).reshape(B, H, M))


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    e, d, G, H, page, B = (4 if c["dtype"] == "f32" else 2), c["head"], c["kv_heads"], c["heads"], c["page"], c["batch"]
    row = G * d * e                                                  # K alone
    if c["kind"] == "bounds":
        pages = sum(max(n // page - max(n - c["new"], 0) // page, 0) for n in _spread(B, c["rows"]))
        return dict(bytes=pages * (page + 2) * row + 4 * pages + 12 * B, flops=2 * pages * page * G * d)
    M, T = c["queries"], c["drafted"]
    if c["kind"] == "shared":
        first, shared, mine = _group_first(c), _prefixes(c), _spread(B, c["suffix"])
        once = sum(shared) + sum(mine) + B * T
        seen = sum(n * (first[g + 1] - first[g]) for g, n in enumerate(shared)) + sum(mine) + B * T
        return dict(bytes=once * 2 * row + 2 * B * M * H * d * e + 4 * B * M * H + 4 * once // page + 4 * B * M * _pages(T, 32),
                    flops=4 * d * H * M * seen)
    spans = [(n, *_candidates(c, n)) for n in _spread(B, c["rows"])]
    if c["kind"] == "select":
        pages = sum(hi - lo for _, lo, hi in spans)
        return dict(bytes=pages * (2 * row + 4) + B * M * H * d * e + 4 * B * G * c["pages"], flops=2 * d * H * M * pages)
    seen = sum(n - (hi - lo) * page + min(c["pages"], hi - lo) * page + T for n, lo, hi in spans)
    return dict(bytes=seen * 2 * row + 2 * B * M * H * d * e + 4 * B * M * H + 4 * G * seen // page + 4 * B * M * _pages(T, 32),
                flops=4 * d * H * M * seen)


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"shared": _exact_shared, "bounds": _exact_bounds, "select": _exact_select, "blocks": _exact_blocks}[case["kind"]](case, st)


def _attend_rows(st, c, slot_of, ids, heads):
    """The softmax over the rows ids[i] of slots slot_of[i] for some kv heads, as a function of a query."""
    cache, page, rep = st["cache"], c["page"], c["heads"] // c["kv_heads"]
    j = torch.tensor(ids, device="cuda")
    s = torch.tensor(slot_of, device="cuda")
    number = cache["table"][s, torch.div(j, page, rounding_mode="floor")].long()
    k = cache["k"][number, j % page][:, heads].double().transpose(0, 1)
    v = cache["v"][number, j % page][:, heads].double().transpose(0, 1)

    def one(q):
        x = torch.bmm(q.double().view(-1, rep, q.shape[-1])[heads], k.transpose(1, 2).contiguous()) * q.shape[-1] ** -0.5
        z = torch.logsumexp(x, -1, keepdim=True)
        return torch.bmm(torch.exp(x - z), v).flatten(0, 1), z.flatten()
    return one


def _drafted(st, b, m, nt, T):
    words = st["tree"][b, m].tolist() if T else []
    return [nt + t for t in range(T) if (words[t // 32] >> (t % 32)) & 1]


def _exact_shared(c, st):
    B, M, H, d = st["q"].shape
    o = torch.zeros(B, M, H, d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, M), float("-inf"), dtype=torch.float64, device="cuda")
    slots, heads = st["slots"].tolist(), list(range(c["kv_heads"]))
    for g, n in enumerate(st["shared"]):
        lead = slots[st["first"][g]]
        for b in range(st["first"][g], st["first"][g + 1]):
            nt = st["true"][b]
            for m in range(M):
                if m == 0 or c["drafted"]:
                    ids = list(range(nt)) + _drafted(st, b, m, nt, c["drafted"])
                    one = _attend_rows(st, c, [lead if j < n else slots[b] for j in ids], ids, heads)
                o[b, m], lse[b, :, m] = one(st["q"][b, m])
    return dict(o=o, lse=lse)


def _exact_bounds(c, st):
    cache, out = st["cache"], st["bounds"].double()
    page, first, lens = c["page"], st["first"].tolist(), cache["lens"].tolist()
    for b, s in enumerate(st["slots"].tolist()):
        row = cache["table"][s].tolist()
        at = [row[i] for i in range(first[b] // page, lens[s] // page)]
        if at:
            ordered = torch.sort(cache["k"][at].double(), 1).values
            out[at, :, 0], out[at, :, 1] = ordered[:, 0], ordered[:, -1]
    return out


def _exact_select(c, st):
    B, M, H, d = st["q"].shape
    G, n = c["kv_heads"], c["pages"]
    out = torch.full((B, G, n), -1, dtype=torch.int64)
    for b, s in enumerate(st["slots"].tolist()):
        lo, hi = _candidates(c, st["true"][b])
        if hi <= lo:
            continue
        number = st["cache"]["table"][s, lo:hi].long()
        best = torch.full((G, hi - lo), float("-inf"), device="cuda")
        for g in range(G):
            low, high = st["bounds"][number, g].double().unbind(1)
            for q in st["q"][b, :, g * (H // G): (g + 1) * (H // G)].reshape(-1, d).double():
                best[g] = torch.maximum(best[g], torch.maximum(low * q, high * q).sum(1).float())
        for g, row in enumerate(best.tolist()):
            mine = sorted(sorted(range(hi - lo), key=lambda i: (-row[i], i))[:n])
            out[b, g, : len(mine)] = torch.tensor(mine) + lo
    return out.to("cuda", torch.int32)


def _exact_blocks(c, st):
    B, M, H, d = st["q"].shape
    page, rep, T = c["page"], H // c["kv_heads"], c["drafted"]
    o = torch.zeros(B, M, H, d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, M), float("-inf"), dtype=torch.float64, device="cuda")
    lists = st["pages"].tolist()
    for b, s in enumerate(st["slots"].tolist()):
        nt = st["true"][b]
        lo, hi = _candidates(c, nt)
        for g in range(c["kv_heads"]):
            listed_ = set(p for p in lists[b][g] if p >= 0)
            rows = [j for p in range(_pages(nt, page)) if p < lo or p >= hi or p in listed_
                    for j in range(p * page, min(nt, (p + 1) * page))]
            for m in range(M):
                if m == 0 or T:
                    ids = rows + _drafted(st, b, m, nt, T)
                    one = _attend_rows(st, c, [s] * len(ids), ids, [g]) if ids else None
                if one:
                    o[b, m, g * rep: (g + 1) * rep], lse[b, g * rep: (g + 1) * rep, m] = one(st["q"][b, m])
    return dict(o=o, lse=lse)
