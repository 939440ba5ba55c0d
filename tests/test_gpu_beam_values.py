"""Beam selection over logits of every size and sign, zeros of both signs among them,
against the fp64 reference: parents and tokens equal, scores within fp32.

A row's total is exact where one logit leaves nothing of the others (the logarithm of
1), and its sum of exponentials is good to 2^-20 otherwise, as for ordinary logits:
what a large value's product with log2(e) loses to rounding is no part of either."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def _run(x, scores, select, finished=None, end=-1):
    import paper_2606_04415_gb300 as fnpu
    g, b, v = x.shape
    ws = torch.full((fnpu.beam_select_workspace(g, b, v, select),), 0xFF, dtype=torch.uint8, device="cuda")
    s, (p, t) = torch.full((g, select), 7.0, device="cuda"), (torch.full((g, select), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    fnpu.beam_select(x.cuda(), scores.cuda(), s, p, t, ws, finished=finished, end_token=end)
    return tuple(a.cpu().numpy() for a in (s, p, t))


def _check(x, scores, select):
    from oracle import pages as P
    s, p, t = _run(x, scores, select)
    ref = P.beam_select(x.float().numpy(), scores.numpy(), None, select, -1)
    assert np.array_equal(p, ref[1]) and np.array_equal(t, ref[2])
    assert (p >= 0).all()
    # one rounding of the total to fp32, and what the sum of exponentials may be off (2^-20 of it)
    off = np.abs(s - ref[0]) - np.abs(ref[0]) * 2.0 ** -24
    assert off.max() <= 2.0 ** -20, "row %d, place %d: %g" % (*np.unravel_index(off.argmax(), off.shape), off.max())


def large(size, sign, dtype, v, seed):
    """Groups of (a row whose logits have that size, an ordinary one): one logit above all
    others, all equal, ordinary values that were shifted there, and a few equal ones above the others."""
    rng = np.random.default_rng([61, seed])
    x = (3 * rng.standard_normal((4, 2, v))).astype(np.float32)
    m = sign * size
    x[0, 0] = m - size * (1 + rng.random(v, dtype=np.float32))
    x[0, 0, v // 3] = m
    x[1, 0] = m
    x[2, 0] += np.float32(m)
    x[3, 0] = 2 * m if sign < 0 else 0
    x[3, 0, 5::v // 7] = m
    return torch.from_numpy(x).to(dtype), torch.from_numpy((-10 * rng.random((4, 2))).astype(np.float32))


SIZES = [1e2, 1e3, 1e4, 3e4, 1e5, 4e5, 1e6, 3e6, 12582912.0, 13002448.0, 3e7, 5e7, 2e8, 1e9, 1e12, 1e20]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", SIZES)
def test_sums_of_large_logits(size, sign, dtype):
    for v in (700, 32000):
        _check(*large(size, sign, dtype, v, seed=v), 6)


@pytest.mark.parametrize("dtype", TYPES)
def test_every_size_beside_every_other(dtype):
    """Rows of one dominating logit: the order of the beams is that of their scores, whatever the logits' size."""
    rows = [sign * s for s in SIZES for sign in (1, -1)]
    x = torch.stack([torch.full((2001,), -1e30 if r < 0 else r - 2 * abs(r)) for r in rows])[None]
    for b, r in enumerate(rows):
        x[0, b, 61 * b] = r
    s = -torch.arange(len(rows), dtype=torch.float32)[None].flip(1) * 2.0 ** -10
    got = _run(x.to(dtype), s, len(rows))
    order = list(range(len(rows)))[::-1]
    assert got[1][0].tolist() == order and got[2][0].tolist() == [61 * b for b in order]
    assert np.abs(got[0][0] - s[0].numpy()[order]).max() <= 2.0 ** -20


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [1, 2, 16, 64])
@pytest.mark.parametrize("v", [40, 3001, 200000])
def test_zeros_of_both_signs_are_equal(v, k, dtype):
    """Ties at zero go to the lowest token, and beams whose zeros have other signs tie."""
    rng = np.random.default_rng([67, v, k])
    x = np.full((3, 4, v), -1.0, np.float32)
    at = np.sort(rng.permutation(v)[:min(v, 2 * k)])
    x[:, :, at] = np.where(rng.random((3, 4, len(at))) < 0.5, np.float32(-0.0), np.float32(0.0))
    x[0, 0, at], x[0, 0, at[-1]] = -0.0, 0.0     # the one that bits would put first stands last
    x[2, :, at[0]] = 2.5                         # zeros below the largest
    s = torch.tensor([[-1.5, -1.5, -1.5, -1.5], [-0.0, 0.0, -0.0, 0.0], [0.0, -0.0, 0.0, 0.0]])
    from oracle import pages as P
    t = torch.from_numpy(x).to(dtype)
    got, ref = _run(t, s, k), P.beam_select(x, s.numpy(), None, k, -1)
    assert np.array_equal(got[1], ref[1]) and np.array_equal(got[2], ref[2])
    assert (np.abs(got[0] - ref[0]) <= np.abs(ref[0]) * 2.0 ** -24 + 2.0 ** -20).all()
    assert not np.signbit(got[0][got[0] == 0]).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_the_lower_zero_is_kept(dtype):
    x = torch.full((1, 1, 64), -1.0)
    x[0, 0, 3], x[0, 0, 9] = -0.0, 0.0
    assert _run(x.to(dtype), torch.zeros(1, 1), 1)[2].tolist() == [[3]]
