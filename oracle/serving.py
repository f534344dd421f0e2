"""Tokens under settings, and contexts that go on in several sequences, in float64 and by walking.

Written from the definitions: the classes of a row sorted by (-logit, index), weights by exp, cuts by running
sums; tables of continuations entry by entry, with a count of who holds each block.
"""
import math

import numpy as np


def choose(l, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(classes that stay, in order; their weights; margin) of one row: margin is how much weight (the largest is 1) the cut of
    top-p is away from moving, inf where top-p is off.  Sums are taken in more than 64 bits."""
    l = np.asarray(l, dtype=np.float64)
    order = np.nonzero(l > -np.inf)[0]
    order = order[np.argsort(-l[order], kind="stable")]
    if temperature == 0:
        return order[:1], np.ones(1), np.inf
    x = (l[order] - l[order[0]]) / float(temperature)
    w = np.exp(x)
    if min_p > 0:
        n = int((x >= math.log(float(min_p))).sum())        # w >= min_p; exp itself would round differences below 2^-53 away
        order, w = order[:n], w[:n]
    if top_k > 0:
        order, w = order[:top_k], w[:top_k]
    margin = np.inf
    if top_p < 1:
        c = np.cumsum(w.astype(np.longdouble))
        need = np.longdouble(top_p) * c[-1]
        n = 1 + int(np.searchsorted(c, need, side="left"))
        n = min(n, len(w))
        margin = min(abs(c[n - 1] - need), abs(need - c[n - 2]) if n > 1 else np.inf)
        order, w = order[:n], w[:n]
    return order, w, float(margin)


def token(l, word, **settings):
    """(token, log of its share, how many stay, margin) of one draw; margin as in choose, of the draw too."""
    order, w, margin = choose(l, **settings)
    u = (int(word) + 0.5) / 2.0 ** 32
    c = np.cumsum(w.astype(np.longdouble))
    t = np.longdouble(u) * c[-1]
    j = min(int(np.searchsorted(c, t, side="right")), len(w) - 1)
    margin = min(margin, abs(c[j] - t), abs(t - c[j - 1]) if j else np.inf)
    x = 0.0 if settings.get("temperature", 1.0) == 0 else (float(l[order[j]]) - float(l[order[0]])) / float(settings.get("temperature", 1.0))
    return int(order[j]), x - math.log(float(c[-1])), len(w), float(margin)


def truncate(l, largest=np.inf, **settings):
    """(row with -inf for what does not stay, how many stay, margin); quotients are held within +-largest."""
    order, _, margin = choose(l, **settings)
    t = float(settings.get("temperature", 1.0))
    out = np.full(len(l), -np.inf)
    out[order] = np.asarray(l, dtype=np.float64)[order] / (t if t > 0 else 1.0)
    out[order] = np.clip(out[order], -largest, largest)
    return out, len(order), margin


def fork(n_blocks, P, table, held, seq_len, src, keep, free, n_free, ld_to):
    """dd_cache_fork: dict of rows (lists of blocks), held, kv_len, free, n_free, moves; "err" where nothing was done."""
    S, n_to = len(held), len(src)
    nothing = dict(err=True, rows=[[] for _ in src], held=[0] * n_to, kv_len=[0] * n_to, free=list(free), n_free=n_free, moves=[])
    if not 0 <= n_free <= n_blocks:
        return nothing
    old = set()
    for q in range(S):
        if not 0 <= held[q] <= len(table[q]) or not 0 <= seq_len[q] <= held[q] * P:
            return nothing
        for b in table[q][:held[q]]:
            if not 0 <= b < n_blocks:
                return nothing
            old.add(int(b))
    rows, lens = [], []
    for s in range(n_to):
        q = src[s]
        if q == -1:
            rows.append([])
            lens.append(0)
            continue
        if not 0 <= q < S:
            return nothing
        k = seq_len[q] if keep is None else keep[s]
        if not 0 <= k <= seq_len[q] or -(-k // P) > ld_to:
            return nothing
        rows.append([int(b) for b in table[q][:-(-k // P)]])
        lens.append(int(k))
    now = {b for r in rows for b in r}
    stack = [int(b) for b in free[:n_free]] + sorted(old - now)
    above = [int(b) for b in free[len(stack):]]
    if len(stack) > n_blocks:
        return nothing
    stays = {}                                    # whose a block is that some sequence has as its partly filled last one
    for s, r in enumerate(rows):
        for j, b in enumerate(r):
            whole = j < len(r) - 1 or lens[s] % P == 0
            stays[b] = min(stays.get(b, n_to), -1 if whole else s)
    lack = [s for s, r in enumerate(rows) if lens[s] % P and stays[r[-1]] != s]
    if len(lack) > len(stack):
        return nothing
    full, moves = list(stack), []
    for s in lack:
        b = stack.pop()
        moves.append((rows[s][-1], b))
        rows[s][-1] = b
    return dict(err=any(not 0 <= b < n_blocks for _, b in moves), rows=rows, held=[len(r) for r in rows], kv_len=lens,
                free=full + above, n_free=len(stack), moves=moves)


def compact(n_blocks, table, held):
    """dd_cache_compact: dict of rows, free (the stack), moves; "err" where nothing was done."""
    rows = [list(t[:max(0, h)]) for t, h in zip(table, held)]
    if any(not 0 <= h <= len(t) for t, h in zip(table, held)) or any(not 0 <= b < n_blocks for r in rows for b in r):
        return dict(err=True)
    used = sorted({int(b) for r in rows for b in r})
    n = len(used)
    holes = [b for b in range(n) if b not in set(used)]
    moves = list(zip([b for b in used if b >= n], holes))
    name = dict(moves)
    return dict(err=False, rows=[[name.get(int(b), int(b)) for b in r] for r in rows], free=list(range(n_blocks - 1, n - 1, -1)), moves=moves)
