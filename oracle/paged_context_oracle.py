"""Float64 definition of the attention over shared and over long contexts in the paged cache: common rows of groups of sequences,
bounds of the keys of every page, the pages that they put first, attention over those.  Plain loops; shares no code with the library.
Caches as in paged_oracle.
"""
import math

import numpy as np

from oracle import paged_oracle as po


def _attend(cache, q, places_of, scale=None):
    """places_of(b, m, g): the (page, row) that query m of entry b sees for kv head g.  As paged_oracle.attend."""
    B, M, H, d = q.shape
    G = cache["k"].shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    o, lse = np.zeros((B, M, H, d)), np.full((B, H, M), -np.inf)
    spread, err = np.zeros((B, M, H, d)), np.zeros((B, H, M))
    for b in range(B):
        for m in range(M):
            for h in range(H):
                g = h // (H // G)
                ids = places_of(b, m, g)
                if not ids:
                    continue
                pages, inner = [p for p, _ in ids], [r for _, r in ids]
                k, v = cache["k"][pages, inner, g], cache["v"][pages, inner, g]
                s = (k @ q[b, m, h]) * scale
                top = s.max()
                if top == -np.inf:
                    continue
                p = np.exp(s - top)
                total = p.sum()
                o[b, m, h] = (p / total) @ v
                spread[b, m, h] = (p / total) @ np.abs(v)
                lse[b, h, m] = top + math.log(total)
                err[b, h, m] = ((np.abs(k) @ np.abs(q[b, m, h])) * scale * (d + 4) * 2.0 ** -24 + np.abs(s) * 2.0 ** -22).max()
    return o, lse, spread, err


def _held(cache, slot, bound):
    n = po.length(cache, slot)
    return n if bound is None else min(n, bound)


def _true(n, n_true, b):
    return n if n_true is None else min(max(n_true[b], 0), n)


def _drafted(tree, b, m, nt, n):
    return [j for j in range(nt, n) if tree is not None and j - nt < tree.shape[2] and tree[b, m, j - nt]]


def groups_of(group_first, B):
    """[(first entry, one past the last)] of each group; an element below the one before it counts as that one."""
    edges, most = [], 0
    for f in group_first:
        most = max(most, min(max(f, 0), B))
        edges.append(most)
    return list(zip(edges, edges[1:]))


def attend_shared(cache, q, group_first, n_shared, *, slots=None, n_true=None, tree=None, scale=None, bound=None):
    B = q.shape[0]
    slots = list(range(B)) if slots is None else slots
    lead = {}
    for g, (lo, hi) in enumerate(groups_of(group_first, B)):
        for b in range(lo, hi):
            lead[b] = (slots[lo], max(n_shared[g], 0))
    seen = {}

    def places(b, m, g):
        if (b, m) not in seen:
            n = _held(cache, slots[b], bound)
            nt = _true(n, n_true, b)
            first, common = lead.get(b, (0, 0))
            of_lead = po.rows_of(cache, first, _held(cache, first, bound)) if common else []
            mine = po.rows_of(cache, slots[b], n) if n else []
            out = [of_lead[j] for j in range(min(common, nt, len(of_lead)))]
            out += [mine[j] for j in range(min(common, nt), nt)] + [mine[j] for j in _drafted(tree, b, m, nt, n)]
            seen[b, m] = [p for p in out if p is not None]
        return seen[b, m]

    return _attend(cache, q, places, scale)


def bounds(cache, before, *, slots, first=None, bound=None):
    """before [P, G, 2, d]."""
    out = before.copy()
    P, page = cache["k"].shape[:2]
    for b, s in enumerate(slots):
        n = _held(cache, s, bound)
        for i in range(n // page):
            p = cache["table"][s][i]
            if (i + 1) * page <= (0 if first is None else max(first[b], 0)) or not 0 <= p < P:
                continue
            for g in range(out.shape[1]):
                for c in range(out.shape[3]):
                    column = [x for x in cache["k"][p, :, g, c] if x == x]
                    out[p, g, 0, c], out[p, g, 1, c] = min(column, default=np.inf), max(column, default=-np.inf)
    return out


def span(nt, window, sinks, page):
    """First page and one past the last that are there to be picked."""
    lead = -(-sinks // page)
    return lead, max(lead, max(nt - window, 0) // page)


def score(q, low, high):
    """q [R, d], low, high [d] -> the score of a page."""
    best = -np.inf
    for row in q:
        total = 0.0
        for x, lo, hi in zip(row, low, high):
            total += x * hi if x > 0 else x * lo if x < 0 else 0.0
        total = float(np.float32(total))
        if total == total:
            best = max(best, total)
    return best


def select(cache, q, bounds, window, sinks, n_select, *, slots=None, n_true=None, bound=None):
    B, M, H, d = q.shape
    P, page, G = cache["k"].shape[:3]
    out = np.full((B, G, n_select), -1)
    for b in range(B):
        s = b if slots is None else slots[b]
        n = _held(cache, s, bound)
        lead, tail = span(_true(n, n_true, b), window, sinks, page)
        for g in range(G):
            rows = q[b, :, g * (H // G): (g + 1) * (H // G)].reshape(-1, d)
            ranked = []
            for i in range(lead, tail):
                p = cache["table"][s][i]
                ranked.append((-score(rows, bounds[p, g, 0], bounds[p, g, 1]) if 0 <= p < P else np.inf, i))
            mine = sorted(i for _, i in sorted(ranked)[:n_select])
            out[b, g, : len(mine)] = mine
    return out


def attend_blocks(cache, q, pages, window, sinks, *, slots=None, n_true=None, tree=None, scale=None, bound=None):
    """pages: lists [B][G][n_select]."""
    page = cache["k"].shape[1]
    seen = {}

    def places(b, m, g):
        if (b, m, g) not in seen:
            s = b if slots is None else slots[b]
            n = _held(cache, s, bound)
            nt = _true(n, n_true, b)
            lead, tail = span(nt, window, sinks, page)
            cols, before, most = [i for i in range(po.pages_of(nt, page)) if i < lead or i >= tail], -1, -1
            for i in list(pages[b][g])[: tail - lead]:
                if i > before and lead <= i < tail and i > most:
                    cols.append(i)
                before = i
                if lead <= i < tail:
                    most = max(most, i)
            mine = po.rows_of(cache, s, n) if n else []
            ids = [j for i in cols for j in range(i * page, min(nt, (i + 1) * page))] + _drafted(tree, b, m, nt, n)
            seen[b, m, g] = [mine[j] for j in ids if mine[j] is not None]
        return seen[b, m, g]

    return _attend(cache, q, places, scale)
