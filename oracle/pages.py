"""Reference for the page operations and the beam selection, row by row.

TEST INFRASTRUCTURE, like the rest of ``oracle``: only ``tests/`` may import
it. It shares no code with the CUDA path. Tables are lists of rows, each the list of
the pages that it holds (-1: freed), so nothing past a row's pages exists here.
"""
from __future__ import annotations

import math

import numpy as np


def held(n, bs):
    return -(-n // bs)


def rows_of(table, length, bs):
    return [[int(e) for e in table[r][:held(int(length[r]), bs)]] for r in range(len(length))]


def free(rows, length, refs, bs, ends=None, window=0, sinks=0):
    """Rows, lengths and counts after pages were given up."""
    rows, length, refs = [list(r) for r in rows], [int(n) for n in length], list(refs)
    for r, row in enumerate(rows):
        end = ends is not None and bool(ends[r])
        for c, e in enumerate(row):
            seen_from = length[r] + 1 - window   # by a query at position `length`
            behind = window > 0 and c * bs >= sinks and (c + 1) * bs <= seen_from
            if e >= 0 and (end or behind):
                refs[e] -= 1
                row[c] = -1
        if end:
            length[r] = 0
    return rows, length, refs


def fork(rows, length, refs, bs, width, parents, grow):
    """(rows, lengths, counts, slots, copies, stats) of the next step."""
    refs = list(refs)
    new = [list(rows[p]) if p >= 0 else [] for p in parents]
    n = [int(length[p]) if p >= 0 else 0 for p in parents]
    for row in rows:
        for e in row:
            if e >= 0:
                refs[e] -= 1
    for row in new:
        for e in row:
            if e >= 0:
                refs[e] += 1
    tail = [new[r][-1] if p >= 0 and grow and n[r] % bs and new[r][-1] >= 0 else None for r, p in enumerate(parents)]
    stuck = [p >= 0 and grow > 0 and (n[r] + grow > width * bs or (n[r] % bs > 0 and new[r][-1] < 0)) for r, p in enumerate(parents)]
    tail = [None if s else t for s, t in zip(stuck, tail)]
    copies_of = []
    for r, t in enumerate(tail):
        same = [i for i, u in enumerate(tail) if u is not None and u == t]
        copies_of.append(t is not None and (refs[t] > len(same) or r != same[0]))
    vacant = [b for b, c in enumerate(refs) if c <= 0]
    need = [0 if p < 0 or stuck[r] else int(copies_of[r]) + held(n[r] + grow, bs) - held(n[r], bs) for r, p in enumerate(parents)]
    at, slots, copies, out_n, taken, unserved = 0, [], [], [], 0, 0
    for r, p in enumerate(parents):
        ids = vacant[at:at + need[r]]
        at += need[r]
        served = p >= 0 and not stuck[r] and len(ids) == need[r]
        pair = [-1, -1]
        if served:
            if copies_of[r]:
                pair = [tail[r], ids[0]]
                refs[tail[r]] -= 1
                new[r][-1] = ids[0]
                new[r] += ids[1:]
            else:
                new[r] += ids
            for b in ids:
                refs[b] = 1
            taken += len(ids)
            pos = range(n[r], n[r] + grow)
            slots.append([new[r][j // bs] * bs + j % bs for j in pos])
        else:
            slots.append([-1] * grow)
            unserved += p >= 0
        out_n.append(n[r] + (grow if served else 0))
        copies.append(pair)
    stats = [len(vacant) - taken, taken, unserved, sum(c[0] >= 0 for c in copies)]
    return new, out_n, refs, slots, copies, stats


def compact(rows, refs, most):
    """(rows, counts, pairs, remap, stats) after moves of live pages to the lowest ids."""
    refs = list(refs)
    live = [b for b, c in enumerate(refs) if c > 0]
    remap = [b if c > 0 else -1 for b, c in enumerate(refs)]
    pairs = []
    for src, dst in zip(reversed(live), [b for b, c in enumerate(refs) if c <= 0]):
        if dst > src or len(pairs) == most:
            break
        pairs.append([src, dst])
        remap[src] = dst
        refs[dst], refs[src] = refs[src], 0
    rows = [[remap[e] if e >= 0 else e for e in row] for row in rows]
    return rows, refs, pairs, remap, [len(live), len(pairs)]


def beam_select(logits, scores, finished, select, end_token):
    """(scores, parents, tokens) [groups, select] of logits [groups, beams, vocab] in fp64."""
    x = np.array(logits, np.float64)
    x[np.isnan(x)] = -np.inf
    x[x == np.inf] = np.finfo(np.float32).max
    g, b, v = x.shape
    out = np.full((g, select), -np.inf), np.full((g, select), -1, np.int64), np.full((g, select), -1, np.int64)
    for i in range(g):
        cands = []
        for j in range(b):
            s = float(scores[i][j])
            if math.isnan(s) or s == -math.inf:
                continue
            if finished is not None and finished[i][j]:
                if end_token >= 0:
                    cands.append((-s, j * v + end_token))
                continue
            m = x[i, j].max()
            if m == -np.inf:
                continue
            with np.errstate(over="ignore"):
                total = s + (x[i, j] - m) - math.log(np.exp(x[i, j] - m).sum())
            best = np.argsort(-x[i, j], kind="stable")[:select]
            cands += [(-total[t], j * v + int(t)) for t in best if x[i, j, t] > -np.inf]
        for k, (t, at) in enumerate(sorted(cands)[:select]):
            out[0][i, k], out[1][i, k], out[2][i, k] = -t, i * b + at // v, at % v
    return out
