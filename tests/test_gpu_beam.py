"""Beam selection against the fp64 reference: parents and tokens equal, scores within
fp32. Inputs are such that no two candidates of different beams are nearer than
1e-5 unless they are equal by construction (a total is good to a few 1e-7 here)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def _run(x, scores, select, finished=None, end=-1, ws=None, out=None):
    import paper_2606_04415_gb300 as fnpu
    g, b, v = x.shape
    if ws is None:
        ws = torch.full((fnpu.beam_select_workspace(g, b, v, select),), 0xFF, dtype=torch.uint8, device="cuda")
    s, p, t = out or (torch.full((g, select), 7.0, device="cuda"), *(torch.full((g, select), 77, dtype=torch.int32, device="cuda") for _ in range(2)))
    fnpu.beam_select(x, scores, s, p, t, ws, finished=finished, end_token=end)
    return s, p, t


def _check(x, scores, select, got, finished=None, end=-1):
    from oracle import pages as P
    s, p, t = (a.cpu().numpy() for a in got)
    ref = P.beam_select(x.float().cpu().numpy(), scores.cpu().numpy(), None if finished is None else finished.cpu().numpy(), select, end)
    assert np.array_equal(p, ref[1]) and np.array_equal(t, ref[2])
    none = p < 0
    assert np.array_equal(s == -np.inf, none)
    # one rounding of the total to fp32, and what the sum of exponentials may be off (2^-20 of it)
    assert (np.abs(s[~none] - ref[0][~none]) <= np.abs(ref[0][~none]) * 2.0 ** -24 + 2.0 ** -20).all()


def _logits(seed, g, b, v, dtype, std=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((g, b, v), device="cuda", generator=gen) * std).to(dtype), -10 * torch.rand((g, b), device="cuda", generator=gen)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("g,b,v,k", [(1, 1, 1, 1), (1, 4, 32000, 8), (3, 5, 50257, 10), (2, 1, 7, 16), (5, 3, 257, 64), (1, 1, 200000, 64),
                                     (40, 8, 1000, 16), (2, 128, 999, 64), (1, 16, 151936, 32), (7, 2, 64, 3)])
def test_select(g, b, v, k, dtype):
    x, s = _logits(g * 1000 + v, g, b, v, dtype)
    _check(x, s, k, _run(x, s, k))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_finished_idle_and_banned(dtype):
    x, s = _logits(5, 6, 4, 5001, dtype)
    x[..., ::7] = -float("inf")
    x[0, 1], x[1] = -float("inf"), -float("inf")      # a row, a group without candidates
    x[2, 0, 5:90], x[2, 1] = float("nan"), float("nan")
    x[3, 2, 17], x[3, 2, 44] = float("inf"), float("inf")
    s[4, 1:], s[5, 2] = -float("inf"), float("nan")
    f = torch.zeros((6, 4), dtype=torch.uint8, device="cuda")
    f[0, 0], f[1, 2], f[2, 3], f[4, 0], f[4, 2] = 1, 1, 255, 1, 1
    for end in (-1, 0, 5000):
        _check(x, s, 9, _run(x, s, 9, f, end), f, end)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("k", [1, 16, 64])
def test_ties_go_to_the_lowest(dtype, k):
    """All logits equal: every slice's candidates are ties, as are those of beams of equal scores."""
    x, s = torch.full((2, 3, 40000), 1.25, dtype=dtype, device="cuda"), torch.full((2, 3), -2.0, device="cuda")
    got = _run(x, s, k)
    assert got[1].tolist() == [[3 * g] * k for g in range(2)] and got[2].tolist() == [list(range(k))] * 2
    x[:, 0, :] = -float("inf")
    x[:, 1, 39990:], x[:, 2, 39990:] = 2.0, 2.0
    got = _run(x, s, k)
    flat = [(b, v) for b in (1, 2) for v in range(39990, 40000)] + [(b, v) for b in (1, 2) for v in range(k)]
    flat = flat[:k] if k <= 20 else flat[:20] + [(1, v) for v in range(k - 20)]
    assert got[1].tolist() == [[3 * g + b for b, _ in flat] for g in range(2)] and got[2].tolist() == [[v for _, v in flat]] * 2


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("period", [1, 8, 256])
def test_large_values_in_few_threads(dtype, period):
    """Ascending and descending rows, and runs of large values, whatever thread holds them."""
    v = 30000
    base = torch.arange(v, device="cuda", dtype=torch.float32) / v
    rows = [base * 40, -base * 40, torch.where(torch.arange(v, device="cuda") // period % 64 == 5, base + 20, base)]
    x = torch.stack(rows)[None].to(dtype).contiguous()
    s = torch.tensor([[0.0, -0.37, -1.03]], device="cuda")
    _check(x, s, 64, _run(x, s, 64))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("g,b,v,off", [(1, 4, 50257, 0), (3, 5, 5003, 3), (40, 8, 9999, 1), (2, 3, 13, 5)])
def test_equal_beams_tie_wherever_their_rows_start(g, b, v, off, dtype):
    """Beams of equal logits and scores have equal totals: the lowest beam's come first, token by token."""
    x, _ = _logits(31, 1, 1, v, dtype)
    buf = torch.zeros(g * b * v + off, dtype=dtype, device="cuda")
    rows = buf[off:].view(g, b, v)
    rows.copy_(x.expand(g, b, v))
    s = torch.full((g, b), -1.5, device="cuda")
    k = min(12, b * v)
    got = _run(rows, s, k)
    flat = x[0, 0].tolist()
    best = sorted(range(v), key=lambda t: (-flat[t], t))[:k]
    want = sorted(((w, t) for t in best for w in range(b)), key=lambda p: (-flat[p[1]], p))  # (equal logits: beams before tokens)
    for i in range(g):
        assert list(zip((got[1][i] - i * b).tolist(), got[2][i].tolist())) == want[:k]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("off,stride", [(0, 5003), (1, 5003), (3, 6007), (5, 8192)])
def test_rows_that_start_anywhere(dtype, off, stride):
    """Slices of a larger buffer whose other values are NaN."""
    buf = torch.full((12 * stride + 16,), float("nan"), device="cuda").to(dtype)
    x, s = _logits(9, 4, 3, 5003, dtype)
    view = torch.as_strided(buf, (4, 3, 5003), (3 * stride, stride, 1), off)
    view.copy_(x)
    _check(x, s, 12, _run(view, s, 12))


def test_scores_far_apart_and_near_each_other():
    """Totals of some hundred whose differences fp32 does not resolve are compared in 64 bits."""
    x = torch.full((1, 4, 300), -30.0, device="cuda")
    x[0, :, 7] = torch.tensor([20.0, 20.0, 20.0, 20.0], device="cuda")
    s = torch.tensor([[-700.0, -700.00006, -700.0, -3.0e30]], device="cuda")
    x[0, 2, 7] = 20.000002       # the rest of its row weighs e^-50: no other effect
    got = _run(x, s, 6)
    assert got[1][0, :3].tolist() == [0, 2, 1] or got[1][0, :3].tolist() == [2, 0, 1]
    _check(x, s, 3, _run(x, s, 3))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits_near_the_ends_of_their_type(dtype):
    """Finite logits whose multiple in base 2 is not, alone and beside ordinary ones."""
    x, s = _logits(13, 4, 2, 3001, dtype)
    x[0, 0, 5], x[0, 0, 2900] = 3e38, 2.5e38
    x[0, 1], x[0, 1, 17:19] = -3e38, -2.9e38
    x[1, 0], x[1, 0, 2000] = -3.3e38, 3.3e38
    x[2, 0, 7], x[2, 0, 8] = float("inf"), 3e38
    x[3, 1] = 3e38
    _check(x, s, 2, _run(x, s, 2))


def test_captured_and_on_other_streams():
    x, s = _logits(21, 2, 4, 20000, torch.bfloat16)
    import paper_2606_04415_gb300 as fnpu
    ws = torch.zeros(fnpu.beam_select_workspace(2, 4, 20000, 8), dtype=torch.uint8, device="cuda")
    out = _run(x, s, 8, ws=ws)
    torch.cuda.synchronize()
    g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=st):
        _run(x, s, 8, ws=ws, out=out)
    for seed in (22, 23):
        y, z = _logits(seed, 2, 4, 20000, torch.bfloat16)
        x.copy_(y), s.copy_(z)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        _check(x, s, 8, out)


@pytest.mark.parametrize("run", [1, 2])
def test_long_slices(run):
    """Rows in one slice each of so many tiles that a thread keeps maxima of several; the reference on the device."""
    g, b, v, k = 61, 5, 130000 * run, 20
    x = torch.randn((g, b, v), device="cuda", generator=torch.Generator(device="cuda").manual_seed(run)) * 3
    s = -10 * torch.rand((g, b), device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))
    got = _run(x, s, k)
    for i in range(0, g, 6):
        total = (s[i].double()[:, None] + torch.log_softmax(x[i].double(), -1)).flatten()
        best = torch.sort(total, descending=True, stable=True)
        assert (got[1][i].long() - i * b).tolist() == (best.indices[:k] // v).tolist()
        assert got[2][i].tolist() == (best.indices[:k] % v).tolist()
        ref = best.values[:k]
        assert ((got[0][i].double() - ref).abs() <= ref.abs() * 2.0 ** -24 + 2.0 ** -20).all()


def test_binding_checks():
    x, s = _logits(3, 2, 4, 100, torch.bfloat16)
    for bad in (lambda: _run(x.half(), s, 4), lambda: _run(x, s.double(), 4), lambda: _run(x, s[:1], 4), lambda: _run(x.transpose(0, 1), s, 4),
                lambda: _run(x[..., ::2], s, 4), lambda: _run(x, s, 4, finished=torch.zeros((2, 4), device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            bad()
    import paper_2606_04415_gb300 as fnpu
    with pytest.raises(fnpu.FnpuError):
        _run(x, s, 4, ws=torch.zeros(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(fnpu.FnpuError):
        _run(x, s, 4, end=100)
