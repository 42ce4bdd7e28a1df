"""Float64 definition of the paged cache's operators: attention of a few queries per sequence over rows in pages, appending
rows, forking sequences, moving the live pages to another pool.  Plain loops over sequences, queries, rows and pages, on a
state of lists and float64 arrays; shares no code with the library.

The cache is a dict: k, v float64 [P, page_rows, G, d]; table [N][W], lens [N], refs [P] lists of whole numbers.
"""
import copy
import math

import numpy as np


def rows_of(cache, slot, n):
    """Place (page, row in page) of the first n rows of a slot; None where the table names no page."""
    P, page = cache["k"].shape[:2]
    out = []
    for j in range(n):
        p = cache["table"][slot][j // page]
        out.append((p, j % page) if 0 <= p < P else None)
    return out


def length(cache, slot):
    if not 0 <= slot < len(cache["lens"]):
        return 0
    return min(max(cache["lens"][slot], 0), len(cache["table"][slot]) * cache["k"].shape[1])


def attend(cache, q, *, slots=None, n_true=None, tree=None, window=0, sinks=0, scale=None, bound=None):
    """q [B, M, H, d]; tree bool [B, M, T] or None.  Returns o, lse and what a float evaluation may be off by:
    spread = sum p |v| of every output, and err = the largest first-order error of a score in float arithmetic."""
    B, M, H, d = q.shape
    G = cache["k"].shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    o, lse = np.zeros((B, M, H, d)), np.full((B, H, M), -np.inf)
    spread, err = np.zeros((B, M, H, d)), np.zeros((B, H, M))
    for b in range(B):
        slot = b if slots is None else slots[b]
        n = length(cache, slot)
        if bound is not None:
            n = min(n, bound)
        nt = n if n_true is None else min(max(n_true[b], 0), n)
        place = rows_of(cache, slot, n) if n else []
        for m in range(M):
            ids = []
            for j in range(n):
                if place[j] is None:
                    continue
                if j < nt:
                    see = window == 0 or j < sinks or j >= nt - window
                else:
                    see = tree is not None and j - nt < tree.shape[2] and tree[b, m, j - nt]
                if see:
                    ids.append(j)
            if not ids:
                continue
            pages, inner = [place[j][0] for j in ids], [place[j][1] for j in ids]
            for h in range(H):
                g = h // (H // G)
                k, v = cache["k"][pages, inner, g], cache["v"][pages, inner, g]
                s = (k @ q[b, m, h]) * scale
                top = s.max()
                p = np.exp(s - top)
                total = p.sum()
                p /= total
                o[b, m, h] = p @ v
                spread[b, m, h] = p @ np.abs(v)
                lse[b, h, m] = top + math.log(total)
                err[b, h, m] = ((np.abs(k) @ np.abs(q[b, m, h])) * scale * (d + 4) * 2.0 ** -24 + np.abs(s) * 2.0 ** -22).max()
    return o, lse, spread, err


def pages_of(rows, page):
    return -(-rows // page)


def rotate(x, pos, base):
    """Rotate-half embedding of one row [G, d] at a position."""
    d = x.shape[-1]
    y = np.array(x, np.float64)
    for c in range(d // 2):
        a = pos * base ** (-2.0 * c / d)
        y[:, c] = x[:, c] * math.cos(a) - x[:, c + d // 2] * math.sin(a)
        y[:, c + d // 2] = x[:, c + d // 2] * math.cos(a) + x[:, c] * math.sin(a)
    return y


def append(cache, k_new, v_new, *, slots=None, pos=None, n_new=None, rope_base=None, positions=None):
    """Returns (cache after, pages missing)."""
    c = copy.deepcopy(cache)
    B, M = k_new.shape[:2]
    P, page = c["k"].shape[:2]
    N, W = len(c["lens"]), len(c["table"][0])
    slots = list(range(B)) if slots is None else list(slots)
    todo, seen = [], set()
    for b in range(B):
        s = slots[b]
        if not 0 <= s < N or s in seen:
            continue
        seen.add(s)
        had = length(c, s)
        at = had if pos is None else min(max(pos[b], 0), had)
        n = M if n_new is None else min(max(n_new[b], 0), M)
        todo.append((b, s, at, n))
        for i in range(pages_of(at, page), pages_of(had, page)):
            p = c["table"][s][i]
            if 0 <= p < P:
                c["refs"][p] -= 1
    shared = []
    for b, s, at, n in todo:
        p = c["table"][s][at // page] if at % page else None
        shared.append(n > 0 and at + n <= W * page and p is not None and (not 0 <= p < P or c["refs"][p] > 1))
    free = [p for p in range(P) if c["refs"][p] <= 0]
    wanted, missing, used = 0, 0, 0
    old = {name: c[name].copy() for name in ("k", "v")}
    for (b, s, at, n), cow in zip(todo, shared):
        if at + n > W * page:
            missing += pages_of(at + n - W * page, page)
            n, cow = 0, False
        need = pages_of(at + n, page) - pages_of(at, page) + cow
        wanted += need
        if need and wanted > len(free):
            c["lens"][s] = at
            continue
        mine = free[wanted - need: wanted]
        if cow:
            p, was = mine.pop(0), c["table"][s][at // page]
            if 0 <= was < P:
                c["refs"][was] -= 1
                for name in ("k", "v"):
                    c[name][p][: at % page] = old[name][was][: at % page]
            c["table"][s][at // page] = p
            c["refs"][p] = 1
        for i, p in enumerate(mine):
            c["table"][s][pages_of(at, page) + i] = p
            c["refs"][p] = 1
        for i in range(n):
            p, r = c["table"][s][(at + i) // page], (at + i) % page
            where = at + i if positions is None else positions[b][i]
            c["k"][p, r] = k_new[b, i] if rope_base is None else rotate(k_new[b, i], where, rope_base)
            c["v"][p, r] = v_new[b, i]
        c["lens"][s] = at + n
    return c, max(wanted - len(free), 0) + missing


def fork(cache, dst, src, rows=None):
    c = copy.deepcopy(cache)
    P, page = c["k"].shape[:2]
    N, W = len(c["lens"]), len(c["table"][0])
    done = set()
    for b in range(len(dst)):
        t, s = dst[b], src[b]
        if not 0 <= t < N or t in done:
            continue
        done.add(t)
        had = length(cache, s)
        n = had if rows is None else min(max(rows[b], 0), had)
        for i in range(pages_of(length(cache, t), page)):
            p = cache["table"][t][i]
            if 0 <= p < P:
                c["refs"][p] -= 1
        c["table"][t] = [cache["table"][s][i] if i < pages_of(n, page) else -1 for i in range(W)]
        for p in c["table"][t][: pages_of(n, page)]:
            if 0 <= p < P:
                c["refs"][p] += 1
        c["lens"][t] = n
    return c


def compact(cache, into):
    c, page = copy.deepcopy(into), cache["k"].shape[1]
    P, Q, W = cache["k"].shape[0], into["k"].shape[0], len(into["table"][0])
    live = [p for p in range(P) if cache["refs"][p] > 0]
    number = {p: i for i, p in enumerate(live) if i < Q}
    for p, i in number.items():
        c["k"][i], c["v"][i] = cache["k"][p], cache["v"][p]
    c["refs"] = [0] * Q
    for s in range(len(cache["lens"])):
        n = length(cache, s)
        held = []
        for i in range(min(pages_of(n, page), W)):
            p = cache["table"][s][i]
            if p not in number:
                break
            held.append(number[p])
        for i in held:
            c["refs"][i] += 1
        c["table"][s] = held + [-1] * (W - len(held))
        c["lens"][s] = min(n, len(held) * page)
    return c, max(len(live) - Q, 0)
