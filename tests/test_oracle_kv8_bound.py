"""The attention bound of the 8-bit cache's reference: a computation whose weights are
rounded once stays within it, and mistakes planted in the reference (a block of values
left out, a scale off by two, two blocks exchanged, nothing at all) do not (no GPU)."""
import math

import numpy as np
import pytest

from oracle import kv8 as K8

FMTS = [K8.INT8, K8.E4M3]


def _bf16(x):
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return (((b + 0x7FFF + ((b >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32).astype(np.float64)


class Case:
    """One sequence of ``n`` keys whose rows vary in size by head and stretch, as in the
    GPU tests, and a few queries that see all of it or less."""

    def __init__(self, n, hq, hkv, d, bs, fmt, q, seed, spread=1.0):
        rng = np.random.default_rng(seed)
        nb = -(-n // bs)
        self.n, self.hq, self.hkv, self.d, self.bs, self.fmt = n, hq, hkv, d, bs, fmt
        self.table = rng.permutation(nb).astype(np.int32)[None]
        pos = np.arange(n)
        sl = self.table[0, pos // bs].astype(np.int64) * bs + pos % bs
        self.pools = [np.zeros(nb * K8.block_bytes(hkv, bs, d), np.uint8) for _ in range(2)]
        for pool in self.pools:
            f = np.exp2(rng.uniform(-spread, spread, (n // 7 + 1, hkv, 1))).repeat(7, 0)[:n]
            K8.append(pool, _bf16(rng.standard_normal((n, hkv, d)) * f), sl, hkv, bs, d, fmt)
        self.q = _bf16(rng.standard_normal((q, hq, d)))

    def reference(self, staged):
        return K8.attention_bound(self.q, [len(self.q)], [self.n], self.table, *self.pools, self.hkv, self.bs, self.d, self.fmt, [staged])

    def out(self, pools, table=None):
        return K8.attention(self.q, [len(self.q)], [self.n], self.table if table is None else table, *pools, self.hkv, self.bs, self.d, self.fmt)[0]


CASES = [(150, 4, 2, 64, 32, 3), (600, 8, 1, 64, 16, 2), (1248, 7, 1, 128, 16, 2), (4174, 4, 2, 64, 32, 2), (6000, 2, 1, 128, 64, 1)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("staged", [False, True])
def test_rounded_weights_stay_within(fmt, case, staged):
    c = Case(*case[:5], fmt, case[5], seed=case[0])
    ref, lse, bound = c.reference(staged)
    assert np.allclose(ref, c.out(c.pools), rtol=1e-12, atol=0)
    pos = np.arange(c.n)
    sl = c.table[0, pos // c.bs].astype(np.int64) * c.bs + pos % c.bs
    k, v = (K8.read(p, sl, c.hkv, c.bs, c.d, fmt) for p in c.pools)
    unit = K8.views(c.pools[1], c.hkv, c.bs, c.d)[1].astype(np.float64)[sl // c.bs]
    G, worst = c.hq // c.hkv, 0.0
    for i in range(len(c.q)):
        see = c.n - len(c.q) + i + 1
        for h in range(c.hq):
            x = (k[:see, h // G] @ c.q[i, h]) / math.sqrt(c.d)
            if staged:
                w = np.exp(x - x.max())
                r, val = _bf16(w), v[:see, h // G]
            else:  # weights with the V scale in their exponent, codes as they are
                e = np.log2(unit[:see, h // G])
                w = np.exp2(x / math.log(2) + e - (x / math.log(2) + e).max())
                r, val = w.astype(np.float16).astype(np.float64), v[:see, h // G] / unit[:see, h // G, None]
                w = w / unit[:see, h // G]
            for total in (w.sum(), r.sum() if staged else (r / unit[:see, h // G]).sum()):
                off = np.abs(_bf16(r @ val / total) - ref[i, h]) / bound[i, h]
                worst = max(worst, off.max())
    assert 0.05 < worst <= 1  # (and the bound is no more than some times what roundings do)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("staged", [False, True])
def test_planted_mistakes_are_seen(fmt, case, staged):
    """Every row shows every mistake, in some of its columns."""
    c = Case(*case[:5], fmt, case[5], seed=case[0])
    ref, _, bound = c.reference(staged)

    def seen(out):
        return (np.abs(_bf16(out) - ref) > bound).any(2)

    assert not seen(ref).any()
    assert seen(np.zeros_like(ref)).all()
    nb = c.table.shape[1]
    for j in (0, nb // 2, nb - 2):
        blk = c.table[0, j]
        for change in ("codes", "scale", "exchange"):
            v, table = c.pools[1].copy(), c.table
            codes, scales = K8.views(v, c.hkv, c.bs, c.d)
            if change == "codes":
                codes[blk] = 128 if fmt == K8.INT8 else 0
            elif change == "scale":
                scales[blk] *= 2
            else:  # the values of a neighbour in their place
                codes[blk], scales[blk] = codes[c.table[0, j + 1]].copy(), scales[c.table[0, j + 1]].copy()
            assert seen(c.out([c.pools[0], v], table)).all(), (j, change)


@pytest.mark.parametrize("fmt", FMTS)
def test_small_blocks_decide_where_the_query_points_at_them(fmt):
    """Blocks 2^30 apart in size and a query on a key of a small one: a bound by the
    row's own weights sees its values, one by the largest value of the cache does not."""
    c = Case(64, 1, 1, 64, 16, fmt, 1, seed=5)
    codes, scales = K8.views(c.pools[1], 1, 16, 64)
    scales[c.table[0, 3]] *= 2.0 ** -30
    k = K8.read(c.pools[0], c.table[0, 3] * 16 + np.arange(15), 1, 16, 64, fmt)[:, 0]
    c.q[0, 0] = _bf16(k[7] * 60)  # (its score is some 500 above the others')
    ref, lse, bound = c.reference(False)
    assert np.abs(ref).max() < 2.0 ** -20 and (bound < 2.0 ** -5 * np.abs(ref).max()).all()
    scales[c.table[0, 3]] *= 2
    assert (np.abs(c.out(c.pools) - ref) > bound).any()
