"""The fp64 reference of rotations and of the 8-bit block cache, against closed
forms, brute force and invariants (no GPU)."""
import math

import numpy as np
import pytest

from oracle import fp8 as F8
from oracle import kv8 as K8

FMTS = [K8.INT8, K8.E4M3]


def test_rope_closed_forms():
    x = np.zeros((3, 1, 4))
    x[:, 0, 0] = 1.0
    f = np.array([math.pi / 2, 0.0], np.float64)
    y = K8.rope(x, [[0, 1, 2]], f)
    want = np.zeros((3, 4))  # (1, 0) turned by 0, a quarter and a half
    want[0, 0], want[1, 2], want[2, 0] = 1, 1, -1
    assert np.allclose(y[:, 0], want, atol=1e-15)
    y = K8.rope(x, [[0, 1, 2]], f, interleaved=True)
    want = np.zeros((3, 4))
    want[0, 0], want[1, 1], want[2, 0] = 1, 1, -1
    assert np.allclose(y[:, 0], want, atol=1e-15)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_invariants(interleaved):
    """Norms are kept, the inverse turns back, and the product of two rotated rows
    depends on the difference of their positions alone."""
    rng = np.random.default_rng(0)
    f = 100.0 ** (-np.arange(6) / 6)
    axis = np.array([0, 0, 1, 1, 2, 2])
    pos = rng.integers(-50, 5000, (3, 7))
    x = rng.standard_normal((7, 2, 16))
    kw = dict(pair_axis=axis, offset=2, interleaved=interleaved)
    y = K8.rope(x, pos, f, **kw)
    assert np.array_equal(y[:, :, :2], x[:, :, :2]) and np.array_equal(y[:, :, 14:], x[:, :, 14:])
    assert np.allclose(np.linalg.norm(y, axis=2), np.linalg.norm(x, axis=2))
    assert np.allclose(K8.rope(y, pos, f, inverse=True, **kw), x)
    z = rng.standard_normal((7, 2, 16))
    shift = np.array([[100], [-3], [7]])
    a = (y * K8.rope(z, pos + 11, f, **kw)).sum(2)
    b = (K8.rope(x, pos + shift, f, **kw) * K8.rope(z, pos + 11 + shift, f, **kw)).sum(2)
    assert np.allclose(a, b)


def test_e4m3_codes_match_the_row_format_reference():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 10, 4000), K8._VALUES[np.isfinite(K8._VALUES)],
                        [448, 464, 480, 1e9, -1e9, 2.0 ** -10, 3 * 2.0 ** -10, 0.0]]).astype(np.float32)
    a, b = K8.encode(x, 0, K8.E4M3), F8.e4m3_round(x)
    same = (a == b) | ((a & 127 == 0) & (b & 127 == 0))  # (the sign of a zero code is free)
    assert same.all()


@pytest.mark.parametrize("fmt", FMTS)
def test_exponent_is_the_least_that_fits(fmt):
    top = K8.LARGEST[fmt]
    for e in (-60, -59, -1, 0, 5, 59, 60):
        assert K8.exponent(math.ldexp(top, e), fmt) == e
        if -60 < e < 60:
            assert K8.exponent(math.nextafter(math.ldexp(top, e), math.inf), fmt) == e + 1
    assert K8.exponent(0.0, fmt) == -60 and K8.exponent(1e-40, fmt) == -60 and K8.exponent(1e38, fmt) == 60


@pytest.mark.parametrize("fmt", FMTS)
def test_append_error_and_growth(fmt):
    """A block filled row by row, each larger than the one before: every row is
    within the errors of its own rounding and of one more for each time that the
    exponent grew; at the end the exponent is the one of the block at once."""
    rng = np.random.default_rng(2)
    hkv, bs, d = 2, 16, 64
    x = rng.standard_normal((bs, hkv, d)) * 1.3 ** np.arange(bs)[:, None, None]
    pool = np.full(3 * K8.block_bytes(hkv, bs, d), 0xFF, np.uint8)
    grew = 0
    last = None
    for i in range(bs):
        K8.append(pool, x[i:i + 1], np.array([16 + i]), hkv, bs, d, fmt)
        sc = K8.views(pool, hkv, bs, d)[1][1].copy()
        grew += last is not None and bool((sc > last).any())
        last = sc
    whole = np.zeros_like(pool)
    K8.append(whole, x, np.arange(16, 32), hkv, bs, d, fmt)
    assert np.array_equal(K8.views(whole, hkv, bs, d)[1][1], last) and grew >= 3
    got = K8.read(pool, np.arange(16, 32), hkv, bs, d, fmt)
    step = last[None, :, None] * (1.0 if fmt == K8.INT8 else 2.0 ** -9)  # spacing of the codes at zero
    bound = step + (0 if fmt == K8.INT8 else 2.0 ** -4 * np.abs(x))
    assert (np.abs(got - x) <= bound).all()
    b = pool.reshape(3, -1)
    assert (b[0] == 0xFF).all() and (b[2] == 0xFF).all()  # the neighbours are untouched


@pytest.mark.parametrize("fmt", FMTS)
def test_attention_against_brute_force_and_paging(fmt):
    """Softmax by hand on a tiny case; permuting the blocks changes nothing; the
    last row of a chunk equals a decode of it."""
    rng = np.random.default_rng(3)
    hq, hkv, bs, d, ctx = 4, 2, 16, 64, 37
    pools = [np.zeros(8 * K8.block_bytes(hkv, bs, d), np.uint8) for _ in range(2)]
    table = np.array([[5, 2, 7]], np.int32)
    pos = np.arange(ctx)
    sl = table[0, pos // bs].astype(np.int64) * bs + pos % bs
    for p in pools:
        K8.append(p, rng.standard_normal((ctx, hkv, d)), sl, hkv, bs, d, fmt)
    q = rng.standard_normal((3, hq, d))
    o, l = K8.attention(q, [3], [ctx], table, *pools, hkv, bs, d, fmt)
    k, v = (K8.read(p, sl, hkv, bs, d, fmt) for p in pools)
    for i in range(3):
        for h in range(hq):
            w = [math.exp(float(np.dot(q[i, h], k[j, h // 2])) / 8) for j in range(ctx - 2 + i)]
            want = sum(wj * v[j, h // 2] for j, wj in enumerate(w)) / sum(w)
            assert np.allclose(o[i, h], want) and math.isclose(l[i, h], math.log(sum(w)), rel_tol=1e-12)
    perm = np.array([3, 0, 6, 1, 7, 2, 5, 4])
    moved = []
    for p in pools:
        m = np.zeros_like(p).reshape(8, -1)
        m[perm] = p.reshape(8, -1)
        moved.append(m.reshape(-1))
    o2, l2 = K8.attention(q, [3], [ctx], perm[table].astype(np.int32), *moved, hkv, bs, d, fmt)
    assert np.array_equal(o, o2) and np.array_equal(l, l2)
    o1, l1 = K8.attention(q[2:], [1], [ctx], table, *pools, hkv, bs, d, fmt)
    assert np.array_equal(o1[0], o[2]) and np.array_equal(l1[0], l[2])
