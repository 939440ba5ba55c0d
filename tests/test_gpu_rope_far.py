"""Rotation at positions past 2^20, to the ends of int32.

Tolerance. The angle in turns is position times inv_freq / 2 pi, kept as two fp32
values f + g, g being the rest of f's product (2^-27.6 inv_freq at most) and the product with the
low half of 1 / (2 pi) (2^-27.2): the errors of g are 2^-24 of the second, 2^-51.2 inv_freq,
and 2^-24 |g|, 2^-50.4 inv_freq, so the angle is within 2^-49.7 * 2 pi < 2^-47 of its own size. To that come a few fp32 roundings of
fractions of a turn (2^-24 of 2 pi each, five at most: 1.9e-6), the functions' 2^-21 and the
rounding of a rotated value to bf16 (2^-8 of it)."""
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


def _cos_sin(pos, f):
    """Cosines and sines of pos * f in fp64: the position in halves of 16 bits, whose
    products with an fp32 value are exact."""
    pos, f = pos.astype(np.int64)[:, None], f.astype(np.float64)[None]
    a, b = ((pos >> 16) << 16).astype(np.float64) * f, (pos & 65535).astype(np.float64) * f
    return np.cos(a) * np.cos(b) - np.sin(a) * np.sin(b), np.sin(a) * np.cos(b) + np.cos(a) * np.sin(b)


def _positions(lo, hi, rng, f):
    """Positions of both signs, among them those whose cosine or sine is smallest: there an
    error of the angle is not hidden by the rounding to bf16."""
    p = np.unique(np.concatenate([rng.integers(lo, hi, 200000), [lo, lo + 1, hi - 1]]))
    c, s = _cos_sin(p, f[:1])
    near = np.argsort(np.minimum(np.abs(c), np.abs(s))[:, 0])[:300]
    p = np.concatenate([p[near], p[:100], p[-100:], [lo, hi - 1]])
    return np.concatenate([p, -p])


RANGES = [(1 << 20, 1 << 24), ((1 << 24) - 5000, (1 << 24) + 5000), (1 << 24, 1 << 27), (1 << 27, 1 << 30), (1 << 30, (1 << 31) - 1)]


@pytest.mark.parametrize("lo,hi", RANGES)
@pytest.mark.parametrize("inv0", [1.0, 0.7310586, 3.1])
@pytest.mark.parametrize("width", [64, 6])
def test_far_positions(lo, hi, inv0, width):
    """Pairs (1, 0): the cosine and the sine themselves, by chunks and pair by pair."""
    import paper_2606_04415_gb300 as fnpu
    rng = np.random.default_rng(hi & 0xFFFF)
    f = (inv0 * 1e3 ** (-np.arange(width // 2) / (width // 2))).astype(np.float32)
    pos = _positions(lo, hi, rng, f)
    if hi == (1 << 31) - 1:
        pos = np.concatenate([pos, [(1 << 31) - 1, -(1 << 31), -(1 << 31) + 1]])
    x = torch.zeros((len(pos), 1, width), dtype=torch.bfloat16)
    x[:, :, :width // 2] = 1
    y = torch.empty_like(x, device="cuda")
    fnpu.rope(fnpu.make_rope(width), torch.from_numpy(f).cuda(), torch.from_numpy(pos.astype(np.int32)[None]).cuda(), x.cuda(), y)
    c, s = _cos_sin(pos, f)
    ref = np.concatenate([c, s], 1)
    size = np.abs(pos.astype(np.float64)[:, None] * f.astype(np.float64)[None])
    tol = 2.0 ** -8 * np.abs(ref) + np.concatenate([size, size], 1) * 2.0 ** -47 + 1.9e-6 + 2.0 ** -21
    off = np.abs(y.double().cpu().numpy()[:, 0] - ref) - tol
    assert (off <= 0).all(), (off.max(), pos[np.unravel_index(off.argmax(), off.shape)[0]])


def test_far_positions_on_the_way_into_a_cache():
    """The same angles in ``rope_append``: queries, and keys read back, equal ``rope``'s."""
    import paper_2606_04415_gb300 as fnpu
    rng = np.random.default_rng(1)
    n, hq, hkv, d, bs = 48, 4, 2, 64, 16
    f = torch.from_numpy((1e4 ** (-np.arange(32) / 32)).astype(np.float32)).cuda()
    pos = rng.integers(-(1 << 31), 1 << 31, n)
    pos[:6] = [(1 << 31) - 1, -(1 << 31), 1 << 24, (1 << 24) + 1, -(1 << 24) - 1, 1 << 30]
    pos = torch.from_numpy(pos.astype(np.int32)).cuda()
    qkv = torch.from_numpy(rng.standard_normal((n, hq + 2 * hkv, d))).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    want = torch.empty((n, hq + hkv, d), dtype=torch.bfloat16, device="cuda")
    fnpu.rope(fnpu.make_rope(d), f, pos, qkv[:, :hq + hkv], want)
    slots = torch.arange(n, device="cuda")
    desc = fnpu.make_desc(hq, hkv, d, d, bs, n // bs)
    for fmt in (fnpu.KV_BF16, fnpu.KV_INT8_BLOCK, fnpu.KV_E4M3_BLOCK):
        size = (n, hkv, d) if fmt == fnpu.KV_BF16 else (n // bs * fnpu.kv8_block_bytes(desc, fmt),)
        pools = [torch.zeros(size, dtype=torch.bfloat16 if fmt == fnpu.KV_BF16 else torch.uint8, device="cuda") for _ in range(2)]
        qo, ko, vo = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda"), *(torch.empty((n, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        fnpu.rope_append(desc, fnpu.make_rope(d), f, pos, q, k, v, slots, qo, *pools, kv_format=fmt)
        fnpu.kv_read(desc, slots, *pools, ko, vo, kv_format=fmt)
        assert torch.equal(qo, want[:, :hq])
        if fmt == fnpu.KV_BF16:
            assert torch.equal(ko, want[:, hq:])
        else:  # within half a step of the codes (rows below 7: int8 steps of 2^-4 at most; e4m3 2^-4 of a value, or 2^-10 of a scale of 2^-6;
            # the rounding of ``want`` to bf16 is 2^-9 of it)
            w = want[:, hq:].float()
            assert ((ko.float() - w).abs() <= (2.0 ** -5 if fmt == fnpu.KV_INT8_BLOCK else 0) + 1.07 * 2.0 ** -4 * w.abs() + 2.0 ** -14).all()
    assert fnpu.check() == fnpu.FNPU_OK
