"""Pins of the references for page operations and beam selection, and what the calls refuse."""
import ctypes
import itertools

import numpy as np
import pytest

import paper_2606_04415_gb300 as fnpu
from oracle import pages as P


def test_fork_by_hand():
    """Blocks of 4; row 0 holds 6 tokens on pages 5, 2, row 1 four on page 7. Two rows
    continue row 0, one row 1, one token more each: row 0's last page is copied for the
    second row, row 1's is full and a block is added. Free: 0, 1, 3, 4, 6."""
    rows, refs = [[5, 2], [7]], [0, 0, 1, 0, 0, 1, 0, 1]
    new, n, refs, slots, copies, stats = P.fork(rows, [6, 4], refs, 4, 8, [0, 0, 1], 1)
    assert new == [[5, 2], [5, 0], [7, 1]] and n == [7, 7, 5]
    assert refs == [1, 1, 1, 0, 0, 2, 0, 1]
    assert slots == [[10], [2], [4]] and copies == [[-1, -1], [2, 0], [-1, -1]] and stats == [3, 2, 0, 1]


def test_fork_with_a_prefix_held_elsewhere():
    """Blocks of 4, three tokens on page 1, which a prefix holds too: both rows would copy
    it and need a block more. Free: 0, 2, 3: the first is served, the second stays as it was."""
    new, n, refs, slots, copies, stats = P.fork([[1]], [3], [0, 2, 0, 0], 4, 4, [0, 0], 2)
    assert new == [[0, 2], [1]] and n == [5, 3] and refs == [1, 2, 1, 0]
    assert slots == [[3, 8], [-1, -1]] and copies == [[1, 0], [-1, -1]] and stats == [1, 2, 1, 1]


def test_free_by_window():
    """Blocks of 4, window 5, sinks 2, 14 tokens: a query at 14 sees 10 .. 14 and 0, 1: pages 1 goes, 2 (8..11) stays."""
    rows, n, refs = P.free([[3, 1, 0, 2]], [14], [1, 1, 1, 1], 4, None, 5, 2)
    assert rows == [[3, -1, 0, 2]] and n == [14] and refs == [1, 0, 1, 1]
    rows, n, refs = P.free([[3, 1, 0, 2]], [14], [1, 1, 1, 1], 4, [1], 5, 2)
    assert rows == [[-1] * 4] and n == [0] and refs == [0] * 4


def test_compact_by_hand():
    rows, refs, pairs, remap, stats = P.compact([[6, 1], [6, 4]], [0, 1, 0, 0, 1, 0, 2, 0], 9)
    assert pairs == [[6, 0], [4, 2]] and rows == [[0, 1], [0, 2]] and refs == [2, 1, 1, 0, 0, 0, 0, 0]
    assert remap == [-1, 1, -1, -1, 2, -1, 0, -1] and stats == [3, 2]
    assert P.compact([[6, 1]], [0, 1, 0, 0, 1, 0, 2, 0], 1)[2] == [[6, 0]]


@pytest.mark.parametrize("seed", range(20))
def test_pages_keep_their_counts(seed):
    """Random steps: counts are the places that hold a page, rows keep their tokens, nothing is written that another holds."""
    rng = np.random.default_rng(seed)
    bs, blocks, width = int(rng.choice([1, 2, 4])), 40, 12
    rows, n, refs, what = [[]], [0], [0] * blocks, {}
    content = [{}]   # of each row: position -> token
    for step in range(12):
        parents = [int(p) for p in rng.integers(-1, len(rows), rng.integers(1, 5))]
        grow = int(rng.integers(0, 4))
        new, m, refs, slots, copies, stats = P.fork(rows, n, refs, bs, width, parents, grow)
        for src, dst in copies:
            if src >= 0:
                for s in range(bs):
                    what[dst * bs + s] = what.get(src * bs + s)
        content = [dict(content[p]) if p >= 0 else {} for p in parents]
        used = set()
        for r in range(len(parents)):
            for g, slot in enumerate(slots[r]):
                if slot >= 0:
                    assert slot not in used and refs[slot // bs] == 1
                    used.add(slot)
                    what[slot] = content[r][m[r] - grow + g] = (step, r, g)
        rows, n = new, m
        for r, row in enumerate(rows):
            assert len(row) == P.held(n[r], bs)
            assert all(what[row[j // bs] * bs + j % bs] == content[r][j] for j in range(n[r]))
        assert refs == np.bincount([e for row in rows for e in row], minlength=blocks).tolist()
        assert stats[0] == refs.count(0)


def test_beam_select_by_brute_force():
    rng = np.random.default_rng(3)
    x, s = rng.standard_normal((2, 3, 7)), rng.standard_normal((2, 3))
    x[0, 1, 3], x[1, 2] = -np.inf, np.nan
    f = np.array([[0, 0, 1], [0, 1, 0]])
    got = P.beam_select(x, s, f, 9, 5)
    for g in range(2):
        cands = []
        for b, v in itertools.product(range(3), range(7)):
            if f[g, b]:
                if v == 5:
                    cands.append((s[g, b], -b, -v))
            elif x[g, b, v] > -np.inf:
                cands.append((s[g, b] + x[g, b, v] - np.log(np.exp(x[g, b][x[g, b] > -np.inf]).sum()), -b, -v))
        cands.sort(reverse=True)
        for k in range(9):
            if k < len(cands):
                assert np.isclose(got[0][g, k], cands[k][0]) and got[1][g, k] == g * 3 - cands[k][1] and got[2][g, k] == -cands[k][2]
            else:
                assert (got[0][g, k], got[1][g, k], got[2][g, k]) == (-np.inf, -1, -1)


# --------------------------------------------------------------- refusals

A = 1 << 20   # an address that nothing reads: the calls are refused before


def _select(dtype=0, stride=100, ws=A, size=1 << 30, logits=A, scores=A, groups=2, beams=3, vocab=100, select=4, end=-1):
    d = fnpu.BeamDesc(groups, beams, vocab, select, dtype, end)
    return fnpu.load().fnpu_beam_select(ctypes.byref(d), logits, stride, scores, None, A, A, A, ws, size, None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(stride=99), dict(ws=None), dict(ws=A + 8), dict(size=64), dict(logits=A + 1), dict(scores=None),
                                dict(dtype=1, logits=A + 2), dict(groups=-1), dict(beams=0), dict(vocab=0), dict(select=0), dict(end=100),
                                dict(end=-2)])
def test_beam_select_refuses(kw):
    assert _select(**kw) == fnpu.FNPU_EINVAL


@pytest.mark.parametrize("kw", [dict(beams=129), dict(select=65), dict(vocab=(1 << 24) + 1, stride=1 << 25)])
def test_beam_select_limits(kw):
    assert _select(**kw) == fnpu.FNPU_EUNSUPPORTED


def _fork(bs=16, blocks=8, rows=2, width=4, new=3, grow=1, table=A, new_table=2 * A, parents=A, slots=A, ws=A, size=1 << 20, stats=A, length=A,
          new_length=2 * A):
    d = fnpu.PagesDesc(bs, blocks)
    return fnpu.load().fnpu_pages_fork(ctypes.byref(d), table, length, rows, width, parents, new, grow, A, new_table, new_length, slots, A, stats,
                                       ws, size, None)


@pytest.mark.parametrize("kw", [dict(bs=0), dict(blocks=0), dict(rows=-1), dict(new=-1), dict(grow=-1), dict(parents=None), dict(new_table=A),
                                dict(new_length=A), dict(slots=None), dict(slots=A + 4), dict(ws=None), dict(size=100), dict(stats=None),
                                dict(table=A + 2), dict(width=-1)])
def test_fork_refuses(kw):
    assert _fork(**kw) == fnpu.FNPU_EINVAL


@pytest.mark.parametrize("kw", [dict(rows=8193), dict(new=8193), dict(grow=(1 << 16) + 1), dict(bs=(1 << 16) + 1), dict(width=1 << 28)])
def test_fork_limits(kw):
    assert _fork(**kw) == fnpu.FNPU_EUNSUPPORTED


def test_other_page_calls_refuse():
    lib, d = fnpu.load(), fnpu.PagesDesc(16, 8)
    ref = ctypes.byref(d)
    assert lib.fnpu_pages_free(ref, A, A, 2, 4, None, -1, 0, A, None) == fnpu.FNPU_EINVAL
    assert lib.fnpu_pages_free(ref, A, A, 2, 4, None, 5, -1, A, None) == fnpu.FNPU_EINVAL
    assert lib.fnpu_pages_free(ref, None, A, 2, 4, None, 5, 0, A, None) == fnpu.FNPU_EINVAL
    assert lib.fnpu_pages_free(ref, A, A, 2, 4, None, 0, 0, A, None) == fnpu.FNPU_OK      # nothing to do
    assert lib.fnpu_pages_compact(ref, A, A, 2, 4, A, None, 3, A, A, A, 1 << 20, None) == fnpu.FNPU_EINVAL
    assert lib.fnpu_pages_compact(ref, A, A, 2, 4, A, A, 3, A, A, A, 64, None) == fnpu.FNPU_EINVAL
    with pytest.raises(fnpu.FnpuError):
        fnpu.pages_workspace(fnpu.make_pages(0, 3), 1)


def test_copy_blocks_refuses():
    lib = fnpu.load()

    def rc(desc, fmt=0, n=2, pools=1, copies=A, k=A, v=A):
        p = ctypes.c_void_p * 1
        return lib.fnpu_kv_copy_blocks(ctypes.byref(desc), fmt, copies, n, p(k), p(v), pools, None)

    d = fnpu.make_desc(4, 2, 64, 64, 16, 8)
    for kw in (dict(fmt=3), dict(n=-1), dict(pools=-1), dict(copies=None), dict(copies=A + 2), dict(k=None), dict(k=A + 8), dict(v=None)):
        assert rc(d, **kw) == fnpu.FNPU_EINVAL
    assert rc(d, n=0) == fnpu.FNPU_OK and rc(d, pools=0) == fnpu.FNPU_OK
    assert rc(fnpu.make_desc(4, 2, 64, 64, 24, 8), fmt=1) == fnpu.FNPU_EUNSUPPORTED
    assert rc(fnpu.make_desc(4, 2, 64, 64, 16, 8, kv_fp8=True)) == fnpu.FNPU_EUNSUPPORTED
