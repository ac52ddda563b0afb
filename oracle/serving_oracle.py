"""CPU oracle for the calls around the verification step: a cache in pages and the draw of tokens.  TEST INFRASTRUCTURE ONLY.

Plain numpy in float64, loops where a definition has them, no code shared with the GPU library.  Pins
(tests/test_oracle_serving.py): attention over pages equals the tree oracle on the gathered cache and a library's causal attention,
a chain given as a tree equals a chain, a window of everything equals none; slots against a dictionary of positions; draws
against a library's sampling filters written another way, and the frequencies of many uniforms.
"""
from __future__ import annotations

import math

import numpy as np

F64 = np.float64


def paged_slots(seq_len, new_len, table, free_pages, free_count, page, max_tokens, source=None):
    """Rows in order take pages from the end of the free list; a row without room gets nothing.

    Returns dict(q_off, slot_map, position, source, table, seq_len, free_count, refused[S]).  source: a list of packed indices per
    row (-1: an entry that is skipped), or None for the tokens' own."""
    table = np.array(table, copy=True)
    rows, width = table.shape
    off, end = [0], 0
    for n in new_len:
        end += max(int(n), 0)
        off.append(min(end, max_tokens))
    slot, pos, src = (np.full(max_tokens, -1, np.int64) for _ in range(3))
    after, refused, asked, taken, begin = [], [], 0, 0, 0
    for s in range(rows):
        length, n = int(seq_len[s]), int(new_len[s])
        begin = sum(max(int(x), 0) for x in new_len[:s])
        ok = n >= 0 and length >= 0 and begin + n <= max_tokens and length + n <= width * page
        have, need = (length + page - 1) // page, 0
        if ok:
            need = (length + n + page - 1) // page - have
            asked += need
            if need and asked > free_count:
                ok = False
            elif need:
                for j in range(need):
                    table[s, have + j] = free_pages[free_count - 1 - taken - j]
                taken += need
        for j in range(max(n, 0)):
            t = begin + j
            if t >= max_tokens:
                break
            pos[t] = max(length, 0) + j
            src[t] = t if source is None else source[s][j]
            if ok and src[t] >= 0:
                slot[t] = table[s, pos[t] // page] * page + pos[t] % page
        after.append(length + n if ok else length)
        refused.append(not ok)
    return dict(q_off=np.array(off), slot_map=slot, position=pos, source=src, table=table, seq_len=np.array(after), free_count=free_count - taken,
                refused=np.array(refused))


def visible(prefix, n_new, parent=None, window=0, n_sink=0):
    """Which of the prefix + n_new keys each new token attends: bool [n_new, prefix + n_new]."""
    sees, depth = np.zeros((n_new, n_new), bool), np.zeros(n_new, np.int64)
    for i in range(n_new):
        if parent is None:
            sees[i, :i + 1], depth[i] = True, i
        else:
            a = i
            while a >= 0:
                sees[i, a] = True
                a = int(parent[a])
            depth[i] = sees[i].sum() - 1
    x, y = prefix + depth, np.concatenate([np.arange(prefix), prefix + depth])
    sees = np.concatenate([np.ones((n_new, prefix), bool), sees], 1)
    if window:
        sees &= (x[:, None] - y[None] < window) | (y[None] < n_sink)
    return sees


def attention(q, k, v, sees, scale=None):
    """One head: q [T,D], k / v [n,D], sees [T,n].  Returns (out, lse, softmax @ |v|, largest sum of |q_d k_d| that a token meets)."""
    q, k, v = (np.asarray(x, F64) for x in (q, k, v))
    scale = scale or 1.0 / math.sqrt(q.shape[1])
    T = len(q)
    out, mag, lse, size = np.zeros((T, q.shape[1])), np.zeros((T, q.shape[1])), np.full(T, -np.inf), np.zeros(T)
    if T == 0:
        return out, lse, mag, size
    if np.isfinite(k).all() and np.isfinite(v).all():
        z = np.where(sees, q @ k.T * scale, -np.inf)
        m = z.max(1, keepdims=True)
        w = np.exp(z - m)
        total = w.sum(1, keepdims=True)
        return w @ v / total, (m + np.log(total))[:, 0], w @ np.abs(v) / total, np.where(sees, np.abs(q) @ np.abs(k).T * scale, 0).max(1)
    with np.errstate(invalid="ignore"):
        for i in range(T):
            at = np.flatnonzero(sees[i])
            z = k[at] @ q[i] * scale
            w = np.exp(z - z.max())
            out[i], mag[i] = (w[:, None] * v[at]).sum(0) / w.sum(), (w[:, None] * np.abs(v[at])).sum(0) / w.sum()
            lse[i], size[i] = z.max() + math.log(w.sum()), (np.abs(k[at]) @ np.abs(q[i]) * scale).max()
    return out, lse, mag, size


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: (token, probability, number of kept entries)."""
    x = np.asarray(logits, F64)
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return -1, 0.0, 0
    if not temperature > 0:
        return int(np.flatnonzero(x == top)[0]), 1.0, 1
    if top == np.inf:
        w = (x == np.inf).astype(F64)
        x = np.where(x == np.inf, 0.0, -np.inf)
    else:
        with np.errstate(over="ignore"):
            w = np.exp((x - top) / temperature)
    keep = x > -np.inf
    if 0 < top_k < len(x):
        keep &= x >= np.sort(x)[::-1][top_k - 1]
    if top_p < 1:
        total = w[keep].sum()
        running, least = 0.0, np.inf
        for value in np.unique(x[keep])[::-1]:
            running += w[keep & (x == value)].sum()
            least = value
            if running >= top_p * total:
                break
        keep &= x >= least
    if min_p > 0:
        keep &= w >= min(min_p, 1.0)
    w = np.where(keep, w, 0.0)
    running = np.cumsum(w)
    over = np.flatnonzero(running > u * running[-1])
    token = int(over[0]) if len(over) else int(np.flatnonzero(w)[-1])
    return token, w[token] / running[-1], int(keep.sum())


def attention_mass(q, lse, k, sees, scale=None):
    """One kv head: q [T,G,D] and lse [T,G] of its query heads, k [n,D], sees [T,n].  Returns (weight that each key gathers, the same with each term times
    its sum of |q_d k_d|, scaled, plus |lse|: what an error of the score is relative to)."""
    q, lse, k = (np.asarray(x, F64) for x in (q, lse, k))
    scale = scale or 1.0 / math.sqrt(q.shape[2])
    got, size = np.zeros(len(k)), np.zeros(len(k))
    for j in range(len(q)):
        at = np.flatnonzero(sees[j])
        for g in range(q.shape[1]):
            if not np.isfinite(lse[j, g]) or not len(at):
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                w = np.exp(k[at] @ q[j, g] * scale - lse[j, g])
                size[at] += w * (np.abs(lse[j, g]) + np.abs(k[at]) @ np.abs(q[j, g]) * scale)
            got[at] += w
    return got, size


def evict_places(mass, length, budget, first=0, recent=0):
    """One row of one layer and kv head: which position ends up in each place that remains."""
    f = min(max(first, 0), length)
    r = min(recent, length - f)
    after = max(min(max(budget, 0), length), f + r)
    weight = [-math.inf if math.isnan(x) else float(x) for x in mass[:length]]
    nan = [math.isnan(x) for x in mass[:length]]
    best = sorted(range(f, length - r), key=lambda y: (nan[y], -weight[y], y))[:after - r - f]
    stay = {y for y in best if y < after - r}
    come = sorted(y for y in best if y >= after - r)
    place = list(range(f)) + [y if y in stay else None for y in range(f, after - r)] + list(range(length - r, length))
    return [come.pop(0) if y is None else y for y in place]
