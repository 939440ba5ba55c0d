"""Rotary positions on the GPU against the fp64 reference.

Tolerance: an output is rounded once to bf16 (half a unit: 2^-8 of its
magnitude); sums of two fp32 products of a cosine or sine good to 2e-6 (angles to
1e-6 rad, and the functions' own errors) add 4e-6 of the inputs' magnitudes."""
import numpy as np
import pytest

from oracle import kv8 as K8

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def _check(y, x, ref):
    x, y = (t.double().cpu().numpy() for t in (x, y))
    size = np.abs(x).max(axis=2, keepdims=True) * 2
    assert (np.abs(y - ref) <= 2.0 ** -8 * np.abs(ref) + 4e-6 * size).all(), np.abs(y - ref).max()


def _freq(pairs, base=1e4):
    return (base ** (-np.arange(pairs) / pairs)).astype(np.float32)


def _case(n, heads, d, rot, offset=0, axes=1, interleaved=False, inverse=False, seed=0, top=40000, stride=None, shift=0):
    """x [n, heads, d] at element ``shift`` of rows ``stride`` apart."""
    rng = np.random.default_rng(seed)
    stride = heads * d if stride is None else stride
    g = torch.Generator().manual_seed(seed)
    buf = torch.randn(n * stride + shift + 8, generator=g).to(torch.bfloat16).cuda()
    x = buf[shift:shift + n * stride].as_strided((n, heads, d), (stride, d, 1), shift)
    pos = rng.integers(0, top, (axes, n)).astype(np.int32)
    axis = rng.integers(0, axes, rot // 2).astype(np.uint8)
    return buf, x, pos, axis, _freq(rot // 2), dict(offset=offset, interleaved=interleaved, inverse=inverse)


def _run(x, out, pos, axis, f, kw, stream=None):
    import paper_2606_04415_gb300 as fnpu
    d = fnpu.make_rope(2 * len(f), kw["offset"], kw["interleaved"], kw["inverse"], pos.shape[0], axis)
    fnpu.rope(d, torch.from_numpy(f).cuda(), torch.from_numpy(pos).cuda(), x, out, stream=stream)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads,d,rot,offset,axes", [
    (1, 1, 64, 64, 0, 1), (1, 28, 128, 128, 0, 1), (7, 4, 64, 32, 0, 2), (33, 5, 80, 80, 0, 3), (130, 12, 128, 64, 32, 4),
    (19, 3, 72, 72, 0, 2), (5, 2, 10, 6, 1, 1), (11, 1, 576, 64, 512, 1), (3, 2, 256, 256, 0, 3), (4, 7, 96, 16, 80, 1), (2000, 32, 128, 128, 0, 3)])
def test_rope(n, heads, d, rot, offset, axes, interleaved):
    """Every width, whole and partial, aligned and not; out of place and in place."""
    _, x, pos, axis, f, kw = _case(n, heads, d, rot, offset, axes, interleaved, seed=n)
    out = torch.full_like(x, float("nan"))
    _run(x, out, pos, axis, f, kw)
    ref = K8.rope(x.double().cpu().numpy(), pos, f, axis, **kw)
    _check(out, x, ref)
    before = x.clone()
    _run(x, x, pos, axis, f, kw)
    _check(x, before, ref)
    assert torch.equal(x.contiguous().view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("shift,pad", [(0, 0), (0, 24), (8, 8), (1, 0), (0, 3), (3, 5)])
def test_rope_strides(shift, pad):
    """Tokens apart and rows off 16 bytes; nothing beside the rows is written."""
    n, heads, d = 37, 6, 64
    buf, x, pos, axis, f, kw = _case(n, heads, d, 64, axes=2, stride=heads * d + pad, shift=shift, seed=pad + shift)
    before = buf.clone()
    ref = K8.rope(x.double().cpu().numpy(), pos, f, axis, **kw)
    old = x.clone()
    _run(x, x, pos, axis, f, kw)
    _check(x, old, ref)
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask[shift:shift + n * (heads * d + pad)].as_strided((n, heads, d), (heads * d + pad, d, 1), shift)[:] = False
    assert torch.equal(buf[mask], before[mask])


def test_rope_far_and_negative_positions():
    """Positions to 2^20 within the same tolerance (the angle itself is a million
    radians), and negative ones."""
    _, x, pos, axis, f, kw = _case(64, 2, 128, 128, top=1 << 20, seed=5)
    pos[0, :5] = [-1, -1000, -4097, (1 << 20) - 1, 0]
    out = torch.empty_like(x)
    _run(x, out, pos, axis, f, kw)
    _check(out, x, K8.rope(x.double().cpu().numpy(), pos, f, axis, **kw))


def test_rope_gradient():
    """The inverse is the transpose: <dy, rope(x)> = <rope_inverse(dy), x>, and the
    gradient of a scalar function by differences."""
    import paper_2606_04415_gb300 as fnpu
    rng = np.random.default_rng(7)
    n, heads, d = 9, 3, 64
    _, x, pos, axis, f, kw = _case(n, heads, d, 64, axes=3, seed=8)
    dy = torch.from_numpy(rng.standard_normal((n, heads, d))).to(torch.bfloat16).cuda()
    dx = torch.empty_like(dy)
    _run(dy, dx, pos, axis, f, dict(kw, inverse=True))
    ref = K8.rope(dy.double().cpu().numpy(), pos, f, axis, **dict(kw, inverse=True))
    _check(dx, dy, ref)
    # loss(x) = sum(dy * rope(x)) is linear: differences of the reference are exact to rounding
    x64, dy64, h = x.double().cpu().numpy(), dy.double().cpu().numpy(), 1e-3
    for i in rng.integers(0, x64.size, 20):
        e = np.zeros(x64.size)
        e[i] = h
        e = e.reshape(x64.shape)
        diff = ((K8.rope(x64 + e, pos, f, axis, **kw) - K8.rope(x64 - e, pos, f, axis, **kw)) * dy64).sum() / (2 * h)
        got = float(dx.double().cpu().numpy().reshape(-1)[i])
        assert abs(got - diff) <= 2.0 ** -8 * abs(diff) + 1e-5 * np.abs(dy64).max() * 2
    assert fnpu.check() == fnpu.FNPU_OK


def test_rope_stream_and_capture():
    """On another stream than the tensors', and replayed from a graph."""
    _, x, pos, axis, f, kw = _case(50, 4, 128, 128, seed=11)
    import paper_2606_04415_gb300 as fnpu
    d = fnpu.make_rope(128)
    fd, pd, out = torch.from_numpy(f).cuda(), torch.from_numpy(pos).cuda(), torch.empty_like(x)
    ref = K8.rope(x.double().cpu().numpy(), pos, f, None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        fnpu.rope(d, fd, pd, x, out)
    s.synchronize()
    _check(out, x, ref)
    g = torch.cuda.CUDAGraph()
    out.zero_()
    with torch.cuda.graph(g):
        fnpu.rope(d, fd, pd, x, out)
    x.copy_(torch.randn(x.shape).to(torch.bfloat16))
    g.replay()
    torch.cuda.synchronize()
    _check(out, x, K8.rope(x.double().cpu().numpy(), pos, f, None))


def test_binding_refuses_other_shapes():
    import paper_2606_04415_gb300 as fnpu
    _, x, pos, _, f, _ = _case(6, 4, 64, 64)
    d, fd, pd = fnpu.make_rope(64), torch.from_numpy(f).cuda(), torch.from_numpy(pos).cuda()
    for bad in (lambda: fnpu.rope(d, fd[:-1], pd, x), lambda: fnpu.rope(d, fd, pd[:, :-1], x), lambda: fnpu.rope(d, fd, pd, x, x[:, :2]),
                lambda: fnpu.rope(d, fd, pd, x.transpose(0, 1)), lambda: fnpu.rope(d, fd, pd, x[:, ::2]), lambda: fnpu.rope(d, fd, pd, x.cpu()),
                lambda: fnpu.rope(d, fd.double(), pd, x), lambda: fnpu.rope(d, fd, pd.long(), x), lambda: fnpu.rope(d, fd, pd, x.float())):
        with pytest.raises((ValueError, TypeError)):
            bad()


# ---------------------------------------------------- append to a bf16 cache

@pytest.mark.parametrize("hq,hkv,d,bs,axes", [(28, 4, 128, 16, 1), (4, 2, 64, 32, 3), (8, 1, 64, 24, 1), (12, 6, 64, 64, 2)])
@pytest.mark.parametrize("n", [1, 70])
def test_append_bf16(hq, hkv, d, bs, axes, n):
    """Queries and keys rotated, values bit-exact, from slices of one projection's
    output; padding slots skipped and the rest of the pool untouched."""
    import paper_2606_04415_gb300 as fnpu
    rng = np.random.default_rng(n + d)
    blocks = 2 * n // bs + 3
    qkv = torch.from_numpy(rng.standard_normal((n, hq + 2 * hkv, d))).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    slots = rng.permutation(blocks * bs)[:n].astype(np.int64)
    if n > 1:
        slots[3], slots[n - 1] = -1, -7
    pos = rng.integers(0, 20000, (axes, n)).astype(np.int32)
    axis, f = rng.integers(0, axes, d // 2).astype(np.uint8), _freq(d // 2, 1e6)
    kc, vc = (torch.from_numpy(rng.standard_normal((blocks * bs, hkv, d))).to(torch.bfloat16).cuda() for _ in range(2))
    k0, v0 = kc.clone(), vc.clone()
    qo = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda")
    desc, rd = fnpu.make_desc(hq, hkv, d, d, bs, blocks), fnpu.make_rope(d, num_axes=axes, pair_axis=axis)
    fnpu.rope_append(desc, rd, torch.from_numpy(f).cuda(), torch.from_numpy(pos).cuda(), q, k, v, torch.from_numpy(slots).cuda(), qo, kc, vc)
    assert fnpu.check() == fnpu.FNPU_OK
    _check(qo, q, K8.rope(q.double().cpu().numpy(), pos, f, axis))
    ok = np.flatnonzero(slots >= 0)
    _check(kc[slots[ok]], k[ok], K8.rope(k.double().cpu().numpy(), pos, f, axis)[ok])
    assert torch.equal(vc[slots[ok]], v[ok])
    rest = np.setdiff1d(np.arange(blocks * bs), slots)
    assert torch.equal(kc[rest], k0[rest]) and torch.equal(vc[rest], v0[rest])
    # the rows read back, in any order, with padding
    sl = np.concatenate([slots, [-1]])
    ko, vo = (torch.full((n + 1, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fnpu.kv_read(desc, torch.from_numpy(sl).cuda(), kc, vc, ko, vo)
    want_k, want_v = kc[np.maximum(sl, 0)], vc[np.maximum(sl, 0)]
    want_k[sl < 0] = 0
    want_v[sl < 0] = 0
    assert torch.equal(ko, want_k) and torch.equal(vo, want_v)
    # a slot past the pool
    slots[0] = blocks * bs
    fnpu.rope_append(desc, rd, torch.from_numpy(f).cuda(), torch.from_numpy(pos).cuda(), None, k, v, torch.from_numpy(slots).cuda(), None, kc, vc)
    assert fnpu.check() == fnpu.FNPU_EDEVICE_RANGE and fnpu.check() == fnpu.FNPU_OK
    fnpu.kv_read(desc, torch.from_numpy(slots).cuda(), kc, vc, ko[:n], vo[:n])
    assert fnpu.check() == fnpu.FNPU_EDEVICE_RANGE and not ko[0].any()


def test_append_latent_in_place():
    """A latent cache: the last 64 of 576 columns turn, queries in place."""
    import paper_2606_04415_gb300 as fnpu
    rng = np.random.default_rng(3)
    n, hq, d, bs, blocks = 21, 16, 576, 64, 4
    q, k = (torch.from_numpy(rng.standard_normal((n, h, d))).to(torch.bfloat16).cuda() for h in (hq, 1))
    pos, f = np.arange(100, 100 + n, dtype=np.int32)[None], _freq(32)
    slots = rng.permutation(bs * blocks)[:n].astype(np.int64)
    kc = torch.zeros((bs * blocks, 1, d), dtype=torch.bfloat16, device="cuda")
    desc, rd = fnpu.make_desc(hq, 1, d, 512, bs, blocks, latent=True), fnpu.make_rope(64, 512, interleaved=True)
    q0 = q.clone()
    fnpu.rope_append(desc, rd, torch.from_numpy(f).cuda(), torch.from_numpy(pos).cuda(), q, k, None, torch.from_numpy(slots).cuda(), q, kc, None)
    kw = dict(offset=512, interleaved=True)
    _check(q, q0, K8.rope(q0.double().cpu().numpy(), pos, f, **kw))
    _check(kc[slots], k, K8.rope(k.double().cpu().numpy(), pos, f, **kw))
    assert torch.equal(q[:, :, :512], q0[:, :, :512]) and torch.equal(kc[slots][:, :, :512], k[:, :, :512])
    ko = torch.empty((n, 1, d), dtype=torch.bfloat16, device="cuda")
    fnpu.kv_read(desc, torch.from_numpy(slots).cuda(), kc, None, ko, None)
    assert torch.equal(ko, kc[slots]) and fnpu.check() == fnpu.FNPU_OK


def test_append_and_read_refuse_other_shapes_and_types():
    """Before any launch: a narrower slice, 32-bit slots and the like would be read past their end."""
    import paper_2606_04415_gb300 as fnpu
    n, hq, hkv, d = 5, 4, 2, 64
    desc, rd, f = fnpu.make_desc(hq, hkv, d, d, 16, 2), fnpu.make_rope(d), torch.from_numpy(_freq(d // 2)).cuda()
    pos, slots = torch.arange(n, dtype=torch.int32, device="cuda"), torch.arange(n, device="cuda")
    qkv = torch.zeros((n, hq + 2 * hkv, d), dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    kc, vc = (torch.zeros((32, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    qo, ko, vo = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(kc[:n]), torch.empty_like(kc[:n])

    def append(q=q, k=k, v=v, slots=slots, qo=qo, f=f, pos=pos):
        fnpu.rope_append(desc, rd, f, pos, q, k, v, slots, qo, kc, vc)

    for bad in (dict(q=qkv[:, :3]), dict(k=qkv[:, 4:5]), dict(v=qkv[:, 7:]), dict(k=k[:, :, :32]), dict(slots=slots.int()), dict(qo=qo[:, :3]),
                dict(qo=None), dict(qo=qo.half()), dict(k=k[:4]), dict(pos=pos.long()), dict(f=f[:31])):
        with pytest.raises((ValueError, TypeError)):
            append(**bad)
    for bad in ((slots.int(), ko, vo), (slots, ko[:4], vo), (slots, ko, vo[:, :1]), (slots, ko.half(), vo), (slots, ko, vo.float())):
        with pytest.raises((ValueError, TypeError)):
            fnpu.kv_read(desc, bad[0], kc, vc, *bad[1:])
    append()
    fnpu.kv_read(desc, slots, kc, vc, ko, vo)
    assert fnpu.check() == fnpu.FNPU_OK and not qo.any() and not ko.any()


# ------------------------------- few heads: several tokens beside each other in a warp

@pytest.mark.parametrize("n,heads,d,rot,offset,axes,interleaved,inverse", [
    (7301, 4, 80, 80, 0, 2, False, False), (9003, 4, 64, 32, 32, 1, True, False), (8000, 1, 128, 128, 0, 3, False, True),
    (7777, 8, 64, 64, 0, 1, False, False), (7303, 2, 40, 8, 4, 2, False, True), (7301, 3, 576, 64, 512, 1, True, False)])
def test_rope_many_tokens_of_few_heads(n, heads, d, rot, offset, axes, interleaved, inverse):
    _, x, pos, axis, f, kw = _case(n, heads, d, rot, offset, axes, interleaved, inverse, seed=n, stride=heads * d + 8)
    out = torch.full((n, heads, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    _run(x, out, pos, axis, f, kw)
    _check(out, x, K8.rope(x.double().cpu().numpy(), pos, f, axis, **kw))
    _run(x, x, pos, axis, f, kw)  # in place
    assert torch.equal(x, out)


@pytest.mark.parametrize("hq,hkv,d,bs,n", [(4, 2, 64, 16, 6401), (8, 1, 64, 32, 7003), (1, 1, 128, 16, 6500)])
def test_append_bf16_many_tokens_of_few_heads(hq, hkv, d, bs, n):
    import paper_2606_04415_gb300 as fnpu
    rng = np.random.default_rng(n)
    blocks = n // bs + 2
    g = torch.Generator(device="cuda").manual_seed(n)
    qkv = torch.randn((n, hq + 2 * hkv, d), device="cuda", generator=g).to(torch.bfloat16)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    slots = rng.permutation(blocks * bs)[:n].astype(np.int64)
    slots[rng.integers(0, n, 50)] = -1
    pos, f = rng.integers(0, 30000, (1, n)).astype(np.int32), _freq(d // 2)
    kc, vc = (torch.randn((blocks * bs, hkv, d), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    k0, v0 = kc.clone(), vc.clone()
    qo = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda")
    args = (fnpu.make_desc(hq, hkv, d, d, bs, blocks), fnpu.make_rope(d), torch.from_numpy(f).cuda(), torch.from_numpy(pos).cuda(), q, k, v)
    fnpu.rope_append(*args, torch.from_numpy(slots).cuda(), qo, kc, vc)
    assert fnpu.check() == fnpu.FNPU_OK
    _check(qo, q, K8.rope(q.double().cpu().numpy(), pos, f))
    ok = np.flatnonzero(slots >= 0)
    _check(kc[slots[ok]], k[ok], K8.rope(k.double().cpu().numpy(), pos, f)[ok])
    assert torch.equal(vc[slots[ok]], v[ok])
    rest = np.setdiff1d(np.arange(blocks * bs), slots)
    assert torch.equal(kc[rest], k0[rest]) and torch.equal(vc[rest], v0[rest])
    slots[n - 1] = blocks * bs  # past the pool
    fnpu.rope_append(*args, torch.from_numpy(slots).cuda(), qo, kc, vc)
    assert fnpu.check() == fnpu.FNPU_EDEVICE_RANGE and fnpu.check() == fnpu.FNPU_OK
