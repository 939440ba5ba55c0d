"""The cache class and the serving loop built of it.

The loop compares an 8-bit cache with a bf16 one on the same rows. Both round
keys (bf16: 2^-8 of each at most) and outputs; the 8-bit codes of N(0, 1) rows are
off by half a step, a uniform error: int8 at most amax / 64 / 2 (the scale is a
power of two: up to 2 amax / 127) with amax below 5, 0.0225 in the root mean square
of keys and values; e4m3 2^-4 of each value, uniform, 0.026 in the root mean
square. A score q.k / sqrt(d) is then off by as much in the root mean square, an
output by that through the weights and through the values: 1.5 times sqrt(2) times
the larger of the two is the bound for a whole step's outputs in the 2-norm."""
import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BOUND = 1.5 * 2 ** 0.5 * 0.026


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def _loop():
    spec = importlib.util.spec_from_file_location("rotary_cache_loop", os.path.join(ROOT, "examples", "rotary_cache_loop.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("heads,block", [((28, 4, 128), 16), ((4, 2, 64), 32)])
def test_serving_loop(fmt, heads, block):
    worst = _loop().main(["--format", fmt, "--heads", *map(str, heads), "--block", str(block), "--sequences", "4", "--prompt", "300",
                          "--chunk", "128", "--tokens", "12"])
    assert 0 < worst <= BOUND


def test_read_gives_what_append_stored():
    """Keys rotated, values as they are, back through ``read``: exact in a bf16 cache."""
    import paper_2606_04415_gb300 as fnpu
    from paper_2606_04415_gb300.rotary import RotaryCache
    g = torch.Generator(device="cuda").manual_seed(1)
    n, f = 40, torch.from_numpy((1e4 ** (-np.arange(32) / 32)).astype(np.float32)).cuda()
    qkv = torch.randn((n, 8, 64), device="cuda", generator=g).to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    slots = torch.arange(16, 16 + n, device="cuda")
    c = RotaryCache(4, 2, 64, 16, 5, fnpu.make_rope(64), f)
    q = c.append(qkv, pos, slots)
    k, v = c.read(slots)
    want = qkv[:, :6].contiguous()
    fnpu.rope(fnpu.make_rope(64), f, pos, want)
    assert torch.equal(q, want[:, :4]) and torch.equal(k, want[:, 4:]) and torch.equal(v, qkv[:, 6:])


@pytest.mark.parametrize("raw", [False, True])
def test_outputs_belong_to_the_stream_that_writes_them(raw):
    """Memory that the caching allocator has back from the current stream, whose last
    writer still waits there, is not the output of a call on another stream."""
    import paper_2606_04415_gb300 as fnpu
    from paper_2606_04415_gb300.rotary import RotaryCache
    g = torch.Generator(device="cuda").manual_seed(2)
    n, f = 300, torch.from_numpy((1e4 ** (-np.arange(32) / 32)).astype(np.float32)).cuda()
    qkv = torch.randn((n, 8, 64), device="cuda", generator=g).to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    slots = torch.arange(n, device="cuda")
    c = RotaryCache(4, 2, 64, 16, 20, fnpu.make_rope(64), f, fnpu.KV_INT8_BLOCK)
    table = np.arange(20, dtype=np.int32)[None]
    plan = c.plan(np.array([n]), np.array([n]), np.array([0]), table)
    want_q = c.append(qkv, pos, slots)
    want = (want_q, *c.attend(plan, want_q), *c.read(slots))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)  # the current stream is busy for some 50 ms
    for t in want:
        x = torch.empty_like(t)
        x.fill_(7)
        del x
    stream = side.cuda_stream if raw else side
    q = c.append(qkv, pos, slots, stream=stream)
    got = (q, *c.attend(plan, q, stream=stream), *c.read(slots, stream=stream))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
