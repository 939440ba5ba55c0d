"""The 8-bit block cache on the GPU against the fp64 reference: append (bit-exact
for rows that do not turn), rows read back, and attention.

Tolerances. A rotated key is stored within half a step of its exact value (int8:
half the scale; e4m3: 2^-4 of its magnitude, or half the subnormal step) plus the
rotation's 8e-6. Attention: the output is rounded to bf16 once (2^-8 of its
magnitude), and the probabilities to f16 (decode: 2^-11 each, doubled for the sums)
or bf16 (prefill: 2^-8 each, doubled likewise) before they weigh values of at most
vmax; the log-sum-exp sees fp32 scores only: 2e-5 a unit of its size or of 1."""
import numpy as np
import pytest

from oracle import kv8 as K8

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FMTS = [K8.INT8, K8.E4M3]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def _bf16(rng, *shape, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(torch.bfloat16)


class Cache:
    """Pools of stale random bytes (NaN codes and wild scales among them), a block
    table, and both sides' appends."""

    def __init__(self, ctx, hq, hkv, d, bs, fmt, seed, blocks=None):
        self.rng = np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.bs, self.fmt, self.ctx = hq, hkv, d, bs, fmt, np.asarray(ctx, np.int32)
        nb = -(-self.ctx // bs)
        self.blocks = int(nb.sum()) + 3 if blocks is None else blocks
        perm = self.rng.permutation(self.blocks)
        self.table = self.rng.integers(0, self.blocks, (len(ctx), int(nb.max()) + 1)).astype(np.int32)
        at = 0
        for s, n in enumerate(nb):
            self.table[s, :n] = perm[at:at + n]
            at += n
        size = self.blocks * K8.block_bytes(hkv, bs, d)
        self.pools = [self.rng.integers(0, 256, size).astype(np.uint8) for _ in range(2)]
        self.dev = [torch.from_numpy(p).cuda() for p in self.pools]
        import paper_2606_04415_gb300 as fnpu
        self.fnpu = fnpu
        self.desc = fnpu.make_desc(hq, hkv, d, d, bs, self.blocks)

    def slots(self, s, a, b):
        pos = np.arange(a, b)
        return self.table[s, pos // self.bs].astype(np.int64) * self.bs + pos % self.bs

    def rows(self, n, spread=1.0):
        """Rows whose size varies by head and stretch of tokens."""
        f = np.exp2(self.rng.uniform(-spread, spread, (n // 7 + 1, self.hkv, 1))).repeat(7, 0)[:n]
        return torch.from_numpy(self.rng.standard_normal((n, self.hkv, self.d)) * f).to(torch.bfloat16)

    def append(self, k, v, slots, check=True):
        """The same rows on both sides; the pools' bytes must agree (e4m3: up to the
        sign of a zero code)."""
        self.fnpu.rope_append(self.desc, None, None, None, None, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda(), None, *self.dev,
                              kv_format=self.fmt)
        for pool, x in zip(self.pools, (k, v)):
            K8.append(pool, x.double().numpy(), slots, self.hkv, self.bs, self.d, self.fmt)
        if check:
            self.same()

    def same(self):
        for name, pool, dev in zip("kv", self.pools, self.dev):
            got = dev.cpu().numpy()
            bad = got != pool
            if self.fmt == K8.E4M3:
                bad &= ((got & 127) != 0) | ((pool & 127) != 0)
            assert not bad.any(), (name, np.flatnonzero(bad)[:8], got[bad][:8], pool[bad][:8])
            pool[:] = got

    def fill(self, upto, spread=1.0):
        """The first upto[s] tokens of every sequence in one call."""
        sl = np.concatenate([self.slots(s, 0, int(n)) for s, n in enumerate(upto)])
        if len(sl):
            self.append(self.rows(len(sl), spread), self.rows(len(sl), spread), sl, check=False)
            self.same()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hkv,d,bs", [(4, 128, 16), (2, 64, 32), (1, 64, 64), (6, 128, 64), (3, 64, 16), (8, 128, 32)])
def test_append_bit_exact(fmt, hkv, d, bs):
    """Whole sequences, then chunks from the middle of a block, then one token at a
    time with growing and shrinking rows: every byte of both pools."""
    c = Cache([bs - 1, 1, 3 * bs + 5, 2 * bs, 70], hkv, hkv, d, bs, fmt, seed=hkv)
    start = [bs // 2, 1, bs + 3, 2 * bs - 1, 20]
    c.fill(start)
    sl = np.concatenate([c.slots(s, a, b) for s, (a, b) in enumerate(zip(start, c.ctx))])
    n = len(sl)
    c.append(c.rows(n, 4.0), c.rows(n, 4.0), sl)  # sizes up to 2^4 apart: scales grow and old rows are stored anew
    for i in range(6):
        one = np.array([c.slots(2, 2 * bs + i, 2 * bs + i + 1)[0], -1, c.slots(4, 64 + i, 65 + i)[0] if i < 6 else -1])
        c.append(c.rows(3) * 3.0 ** i, c.rows(3) * 0.3 ** i, one)
    assert c.fnpu.check() == c.fnpu.FNPU_OK


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d,bs", [(64, 16), (128, 64)])
def test_append_many(fmt, d, bs):
    """More runs than one wave of the grid: thousands of single rows in blocks that
    hold rows already, then one long chunk; and none (zero tokens)."""
    n = 3000 if d == 64 else 1200
    c = Cache([bs] * n, 2, 2, d, bs, fmt, seed=d)
    first = np.concatenate([c.slots(s, 0, 3) for s in range(n)])
    c.append(c.rows(3 * n), c.rows(3 * n), first, check=False)
    c.append(c.rows(n, 4.0), c.rows(n, 4.0), np.array([c.slots(s, 3, 4)[0] for s in c.rng.permutation(n)]))
    long = Cache([5000], 2, 2, d, bs, fmt, seed=d + 1)
    long.fill([7])
    long.append(long.rows(4993), long.rows(4993), long.slots(0, 7, 5000))
    long.append(long.rows(0), long.rows(0), np.zeros(0, np.int64))
    assert c.fnpu.check() == c.fnpu.FNPU_OK


@pytest.mark.parametrize("fmt", FMTS)
def test_append_special_rows(fmt):
    """Zero rows, tiny and huge rows, exact largest values and ties, negative
    zeros; a block begun afresh forgets its scale; padding between runs."""
    c = Cache([64, 64], 4, 4, 128, 16, fmt, seed=9)
    k, v = c.rows(64), c.rows(64)
    k[0:16] = 0
    k[16:32] *= 2.0 ** -100
    k[32:48] *= 2.0 ** 50
    v[0] = -0.0
    v[1:16] = 0
    v[16:32] = torch.arange(128, dtype=torch.float32).to(torch.bfloat16) / 2 - 32
    v[32:48, :, 0] = K8.LARGEST[fmt]
    v[48:64, 1] *= 1e-3
    sl = c.slots(0, 0, 64)
    c.append(k, v, sl)
    c.append(k.flip(0), v.flip(0), sl)                       # fresh blocks again: nothing of before
    c.append(c.rows(16) * 2.0 ** 55, c.rows(16), c.slots(1, 0, 16))
    sl = np.concatenate([c.slots(1, 16, 20), [-1, -1], c.slots(1, 32, 37), [-5]])
    c.append(c.rows(len(sl)), c.rows(len(sl)), sl)
    assert c.fnpu.check() == c.fnpu.FNPU_OK


@pytest.mark.parametrize("fmt", FMTS)
def test_append_not_finite(fmt):
    """NaN is stored as zero, an infinity as the largest value, too large values
    saturate; each raises the flag, and no row but their own block's head is touched."""
    c = Cache([40], 2, 2, 64, 16, fmt, seed=10)
    k, v = c.rows(40), c.rows(40)
    k[3, 0, 5], k[4, 0, 6], v[20, 1, 7] = float("nan"), float("-inf"), 3e38
    sl = c.slots(0, 0, 40)
    c.fnpu.rope_append(c.desc, None, None, None, None, k.cuda(), v.cuda(), torch.from_numpy(sl).cuda(), None, *c.dev, kv_format=fmt)
    assert c.fnpu.check() == c.fnpu.FNPU_EDEVICE_RANGE and c.fnpu.check() == c.fnpu.FNPU_OK
    codes, scales = K8.views(c.dev[0].cpu().numpy(), 2, 16, 64)
    b = c.table[0, 0]
    got = K8.decode(codes[b, 0], fmt) * scales[b, 0]
    fin = k[:16, 0].double().numpy()
    fin[3, 5] = fin[4, 6] = 0
    e = K8.exponent(np.abs(fin).max(), fmt)
    assert scales[b, 0] == 2.0 ** e and got[3, 5] == 0 and got[4, 6] == -K8.LARGEST[fmt] * 2.0 ** e
    fin[4, 6] = -K8.LARGEST[fmt] * 2.0 ** e
    assert np.array_equal(got, K8.decode(K8.encode(fin, e, fmt), fmt) * 2.0 ** e)
    codes, scales = K8.views(c.dev[1].cpu().numpy(), 2, 16, 64)
    b = c.table[0, 1]
    assert scales[b, 1] == 2.0 ** 60 and K8.decode(codes[b, 1, 4, 7], fmt) == K8.LARGEST[fmt] and scales[b, 0] < 1


@pytest.mark.parametrize("fmt", FMTS)
def test_append_out_of_range_slot(fmt):
    c = Cache([30], 2, 2, 64, 16, fmt, seed=11)
    sl = np.concatenate([c.slots(0, 0, 5), [c.blocks * 16, c.blocks * 16 + 1], c.slots(0, 16, 20)])
    k, v = c.rows(len(sl)), c.rows(len(sl))
    c.fnpu.rope_append(c.desc, None, None, None, None, k.cuda(), v.cuda(), torch.from_numpy(sl).cuda(), None, *c.dev, kv_format=fmt)
    assert c.fnpu.check() == c.fnpu.FNPU_EDEVICE_RANGE
    sl[5:7] = -1
    for pool, x in zip(c.pools, (k, v)):
        K8.append(pool, x.double().numpy(), sl, 2, 16, 64, fmt)
    c.same()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs,rot,offset,inter,axes", [(28, 4, 128, 16, 128, 0, False, 1), (4, 2, 64, 32, 64, 0, True, 3),
                                                               (8, 1, 64, 64, 32, 16, False, 2), (12, 6, 128, 64, 64, 64, True, 1)])
def test_rope_append(fmt, hq, hkv, d, bs, rot, offset, inter, axes):
    """Queries, rotated keys within half a step, values bit-exact, in one call on
    slices of one projection's output; then rows read back exactly."""
    c = Cache([bs + 5, 3 * bs, 1, 90], hq, hkv, d, bs, fmt, seed=rot)
    start = [bs - 2, 0, 0, 33]
    c.fill(start)
    sl = np.concatenate([c.slots(s, a, b) for s, (a, b) in enumerate(zip(start, c.ctx))])
    n = len(sl)
    qkv = (_bf16(c.rng, n, hq + 2 * hkv, d) * torch.from_numpy(2.0 ** c.rng.integers(-1, 2, (n, 1, 1)))).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    pos = c.rng.integers(0, 30000, (axes, n)).astype(np.int32)
    axis, f = c.rng.integers(0, axes, rot // 2).astype(np.uint8), (1e4 ** (-np.arange(rot // 2) * 2 / rot)).astype(np.float32)
    rd = c.fnpu.make_rope(rot, offset, inter, num_axes=axes, pair_axis=axis)
    qo = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda")
    c.fnpu.rope_append(c.desc, rd, torch.from_numpy(f).cuda(), torch.from_numpy(pos).cuda(), q, k, v, torch.from_numpy(sl).cuda(), qo, *c.dev,
                       kv_format=fmt)
    assert c.fnpu.check() == c.fnpu.FNPU_OK
    kw = dict(offset=offset, interleaved=inter)
    qr, kr = (K8.rope(x.double().cpu().numpy(), pos, f, axis, **kw) for x in (q, k))
    got = qo.double().cpu().numpy()
    assert (np.abs(got - qr) <= 2.0 ** -8 * np.abs(qr) + 8e-6 * np.abs(q.double().cpu().numpy()).max(2, keepdims=True)).all()
    before = K8.read(c.pools[0], np.concatenate([c.slots(s, 0, a) for s, a in enumerate(start)]), hkv, bs, d, fmt)
    K8.append(c.pools[0], kr, sl, hkv, bs, d, fmt)
    K8.append(c.pools[1], v.double().cpu().numpy(), sl, hkv, bs, d, fmt)
    # keys: the exponents agree (none of these blocks is within 1e-5 of a boundary), values within half a step
    dk = c.dev[0].cpu().numpy()
    scale = K8.views(dk, hkv, bs, d)[1]
    assert np.array_equal(scale[sl // bs], K8.views(c.pools[0], hkv, bs, d)[1][sl // bs])
    st = K8.read(dk, sl, hkv, bs, d, fmt)
    half = scale[sl // bs][:, :, None] * (0.5 if fmt == K8.INT8 else 2.0 ** -10)
    assert (np.abs(st - kr) <= half + (0 if fmt == K8.INT8 else 2.0 ** -4 * np.abs(kr)) + 8e-6 * np.abs(kr).max()).all()
    # rows of before: as stored, or stored anew over a grown scale
    held = np.concatenate([c.slots(s, 0, a) for s, a in enumerate(start)])
    assert np.array_equal(K8.read(dk, held, hkv, bs, d, fmt), K8.read(c.pools[0], held, hkv, bs, d, fmt)) and before.shape[0] == len(held)
    c.pools[0][:] = dk
    c.same()
    all_sl = np.concatenate([c.slots(s, 0, int(n_)) for s, n_ in enumerate(c.ctx)] + [[-1]])[::-1].copy()
    out = [torch.full((len(all_sl), hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    c.fnpu.kv_read(c.desc, torch.from_numpy(all_sl).cuda(), *c.dev, *out, kv_format=fmt)
    for o, pool in zip(out, c.pools):
        assert np.array_equal(o.double().cpu().numpy(), K8.read(pool, all_sl, hkv, bs, d, fmt))
    assert c.fnpu.check() == c.fnpu.FNPU_OK


# -------------------------------------------------------------- attention

def _attend(c, ql, phase=None, q=None, opts=None, plan=None, scale=1.0, spread=1.0, tokens=None, stream=None):
    """Plan, run and compare with the reference; ``c`` holds every key."""
    ql = np.asarray(ql, np.int32)
    phase = (ql == 1).astype(np.uint8) if phase is None else phase
    T = int(ql.sum())
    q = _bf16(c.rng, T, c.hq, c.d, scale=scale).cuda() if q is None else q
    out = torch.full((T, c.hq, c.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, c.hq), float("nan"), device="cuda")
    if plan is None:
        plan = c.fnpu.kv8_attn_plan(c.desc, c.fmt, ql, c.ctx, phase, c.table, opts=opts)
    c.fnpu.mixed_attn_run(plan, q, *c.dev, out, lse)
    assert c.fnpu.plan_check(plan) == c.fnpu.FNPU_OK and c.fnpu.check() == c.fnpu.FNPU_OK
    _compare(c, ql, q, out, lse, tokens)
    return plan, q, out, lse


def _compare(c, ql, q, out, lse, tokens=None):
    ref_o, ref_l = K8.attention(q.double().cpu().numpy(), ql, c.ctx, c.table, *c.pools, c.hkv, c.bs, c.d, c.fmt, tokens=tokens)
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    at = 0
    for s, n in enumerate(ql):
        vmax = np.abs(K8.read(c.pools[1], c.slots(s, 0, int(c.ctx[s])), c.hkv, c.bs, c.d, c.fmt)).max((0, 2)).repeat(c.hq // c.hkv)[:, None]
        short = n * (c.hq // c.hkv) <= 64
        for t in range(at, at + n):
            if tokens is not None and t not in tokens:
                continue
            bad = np.abs(o[t] - ref_o[t]) - (2.0 ** -8 * np.abs(ref_o[t]) + (2.0 ** -10 if short else 2.0 ** -7) * vmax)
            assert (bad <= 0).all(), (s, t - at, bad.max())
            assert (np.abs(l[t] - ref_l[t]) <= 2e-5 * np.maximum(1, np.abs(ref_l[t]))).all(), (s, t - at, np.abs(l[t] - ref_l[t]).max())
        at += n


LAYOUTS = [(28, 4, 128, 16), (4, 2, 64, 32), (8, 1, 64, 16), (32, 8, 128, 64), (6, 3, 128, 32), (12, 6, 64, 64), (16, 16, 64, 16),
           (40, 1, 128, 32), (71, 1, 64, 16), (3, 3, 64, 16), (2, 2, 128, 64)]
RAGGED = [1, 2, 15, 16, 17, 31, 33, 64, 65, 130, 513]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs", LAYOUTS)
def test_decode(fmt, hq, hkv, d, bs):
    c = Cache(RAGGED, hq, hkv, d, bs, fmt, seed=hq + bs)
    c.fill(c.ctx)
    plan, q, out, lse = _attend(c, np.ones(len(RAGGED), np.int32))
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    c.fnpu.mixed_attn_run(plan, q, *c.dev, o2, l2)  # the same plan again: the same bits
    assert torch.equal(o2, out) and torch.equal(l2, lse)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs", [(28, 4, 128, 16), (4, 2, 64, 32), (8, 1, 64, 64), (6, 3, 128, 32)])
@pytest.mark.parametrize("split", [16, 48, 320])
def test_decode_splits(fmt, hq, hkv, d, bs, split):
    """Pieces of a tile, of three (a piece may end inside a block and a stage), and
    of many; several tokens a sequence, so that a piece may have no key for some."""
    import paper_2606_04415_gb300 as fnpu
    ctx = [1, 17, 49, 100, 333, 641, 5, 96]
    ql = [1, 2, 5, 4, 1, 8, 5, 3]
    c = Cache(ctx, hq, hkv, d, bs, fmt, seed=split)
    c.fill(c.ctx)
    _attend(c, ql, opts=fnpu.PlanOpts(split, 0, 0, 0))
    _attend(c, ql, phase=np.zeros(len(ql), np.uint8))


@pytest.mark.parametrize("fmt", FMTS)
def test_decode_scales_far_apart(fmt):
    """Blocks whose keys and values are 2^40 apart in size, all-zero value blocks,
    queries from 2^-30 to 2^30: what a weight of 2^e times a code can lose."""
    c = Cache([200, 333, 64, 18], 8, 2, 128, 16, fmt, seed=21)
    n = int(c.ctx.sum())
    sl = np.concatenate([c.slots(s, 0, int(x)) for s, x in enumerate(c.ctx)])
    k, v = c.rows(n), c.rows(n)
    blockwise = np.exp2(c.rng.integers(-20, 21, (n // 16 + 1, 2, 1))).repeat(16, 0)[:n]
    v = (v.double() * torch.from_numpy(blockwise)).to(torch.bfloat16)
    v[40:64] = 0
    v[np.arange(200, 216)] = 0
    c.append(k, v, sl)
    q = _bf16(c.rng, 4, 8, 128)
    q[0] *= 2.0 ** 20 * 0  # all scores equal
    q[1] *= 8
    q[2] *= 2.0 ** -30
    _attend(c, [1, 1, 1, 1], q=q.cuda())
    k2 = (k.double() * 2.0 ** -30).to(torch.bfloat16)
    c.append(k2, v, sl)
    _attend(c, [1, 1, 1, 1], q=(_bf16(c.rng, 4, 8, 128).double() * 2.0 ** 30).to(torch.bfloat16).cuda())


@pytest.mark.parametrize("fmt", FMTS)
def test_decode_rising_and_falling_scores(fmt):
    """Scores that climb by several units a tile (the running maximum moves all the
    time, by less and by more than its slack) and that fall (it never moves)."""
    c = Cache([300, 300], 4, 2, 64, 32, fmt, seed=22)
    u = np.ones(64) / 8
    for s, sign in ((0, 1), (1, -1)):
        k = torch.from_numpy(sign * np.arange(300)[:, None, None] * u / 6 + 0.01 * c.rng.standard_normal((300, 2, 64))).to(torch.bfloat16)
        c.append(k, c.rows(300), c.slots(s, 0, 300))
    q = torch.from_numpy(np.broadcast_to(u * 8, (2, 4, 64)) * np.array([1, 2, 4, 0.1])[None, :, None]).to(torch.bfloat16).cuda()
    _attend(c, [1, 1], q=q)
    _attend(c, [1, 1], q=q, opts=c.fnpu.PlanOpts(64, 0, 0, 0))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("ql", [1, 3, 9])
def test_query_rows_do_not_mix(fmt, ql):
    """A row of NaN, one with an infinity and one of zeros among others: theirs
    alone are NaN (or plain means); every other row is what it would be."""
    c = Cache([150, 40], 8, 2, 64, 16, fmt, seed=24)
    c.fill(c.ctx)
    T = 2 * ql
    q = _bf16(c.rng, T, 8, 64)
    clean = q.clone()
    q[0, 1], q[ql, 6, 3], q[T - 1, 4] = float("nan"), float("inf"), 0
    clean[T - 1, 4] = 0
    plan, _, o, l = _attend(c, [ql, ql], q=clean.cuda())
    o2, l2 = torch.empty_like(o), torch.empty_like(l)
    c.fnpu.mixed_attn_run(plan, q.cuda(), *c.dev, o2, l2)
    odd = torch.zeros((T, 8), dtype=torch.bool)
    odd[0, 1] = odd[ql, 6] = True
    assert torch.equal(o2.cpu()[~odd], o.cpu()[~odd]) and torch.equal(l2.cpu()[~odd], l.cpu()[~odd])
    assert o2.cpu()[odd].isnan().all() and l2.cpu()[0, 1].isnan()


def test_append_then_attend_across_streams_and_replays():
    """A step captured with its append: replayed for the next token with new rows,
    positions and slots in the same buffers; the append on one stream, the attention on
    another after an event."""
    import paper_2606_04415_gb300 as fnpu
    fmt = K8.INT8
    c = Cache([65, 30], 4, 2, 64, 16, fmt, seed=25)
    c.ctx = c.ctx - 2
    c.fill(c.ctx)
    f = (1e4 ** (-np.arange(32) / 32)).astype(np.float32)
    rd, fd = fnpu.make_rope(64), torch.from_numpy(f).cuda()
    qkv = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    pos, slots = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    q, out, lse = torch.empty((2, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 4), device="cuda")
    plan = fnpu.kv8_attn_plan(c.desc, fmt, [1, 1], c.ctx + 1, [1, 1], c.table)

    def append():
        fnpu.rope_append(c.desc, rd, fd, pos, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], slots, q, *c.dev, kv_format=fmt)

    def put():
        x = _bf16(c.rng, 2, 8, 64)
        qkv.copy_(x)
        pos.copy_(torch.from_numpy(c.ctx[None]))
        slots.copy_(torch.from_numpy(np.array([c.slots(s, int(n), int(n) + 1)[0] for s, n in enumerate(c.ctx)])))
        return x

    def check(x):
        torch.cuda.synchronize()
        assert fnpu.plan_check(plan) == fnpu.FNPU_OK and fnpu.check() == fnpu.FNPU_OK
        sl = slots.cpu().numpy()
        before = K8.views(c.pools[0], 2, 16, 64)[1].copy()
        K8.append(c.pools[0], K8.rope(x[:, 4:6].double().numpy(), pos.cpu().numpy(), f), sl, 2, 16, 64, fmt)
        K8.append(c.pools[1], x[:, 6:].double().numpy(), sl, 2, 16, 64, fmt)
        got = c.dev[0].cpu().numpy()
        assert np.abs(K8.read(got, sl, 2, 16, 64, fmt) - K8.read(c.pools[0], sl, 2, 16, 64, fmt)).max() <= before.max() * 2
        c.pools[0][:] = got
        c.same()
        c.ctx = c.ctx + 1
        _compare(c, [1, 1], q, out, lse)

    x = put()
    s1, s2, e = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.Event()
    s1.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s1):
        append()
        e.record()
    s2.wait_event(e)
    with torch.cuda.stream(s2):
        fnpu.mixed_attn_run(plan, q, *c.dev, out, lse)
    check(x)
    fnpu.mixed_attn_replan(plan, [1, 1], c.ctx + 1, [1, 1], c.table)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        append()
        fnpu.mixed_attn_run(plan, q, *c.dev, out, lse)
    x = put()
    g.replay()
    check(x)


@pytest.mark.parametrize("fmt", FMTS)
def test_long_context(fmt):
    """A context past the cap on splits, beside short ones."""
    c = Cache([40011, 3, 900], 7, 1, 128, 64, fmt, seed=23)
    c.fill(c.ctx)
    _attend(c, [2, 1, 1])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs", [(28, 4, 128, 16), (4, 2, 64, 32), (32, 8, 128, 64), (8, 1, 64, 16)])
def test_mixed(fmt, hq, hkv, d, bs):
    """Chunks on prefixes, short chunks and decodes in one step, co-located and
    with separate launches."""
    import paper_2606_04415_gb300 as fnpu
    ctx, ql = [230, 300, 1, 77, 700, 64, 18], [200, 130, 1, 77, 1, 3, 1]
    c = Cache(ctx, hq, hkv, d, bs, fmt, seed=bs)
    c.fill(c.ctx)
    rows = set(c.rng.permutation(sum(ql))[:60].tolist()) | {0, 199, 200, 329, 330, 331, 408, 409, 412}
    plan, q, out, lse = _attend(c, ql, tokens=rows)
    for opts in (fnpu.PlanOpts(0, 0, 0, fnpu.PLAN_SEPARATE_LAUNCHES), fnpu.PlanOpts(0, 10, 0, 0), fnpu.PlanOpts(0, 20, 0, fnpu.PLAN_GREEN_CONTEXTS)):
        try:
            p2 = fnpu.kv8_attn_plan(c.desc, fmt, np.array(ql), c.ctx, (np.array(ql) == 1).astype(np.uint8), c.table, opts=opts)
        except fnpu.FnpuError as e:
            assert opts.flags == fnpu.PLAN_GREEN_CONTEXTS and e.code == fnpu.FNPU_EUNSUPPORTED
            continue
        o2, l2 = torch.full_like(out, float("nan")), torch.full_like(lse, float("nan"))
        fnpu.mixed_attn_run(p2, q, *c.dev, o2, l2)
        assert fnpu.plan_check(p2) == fnpu.FNPU_OK
        _compare(c, ql, q, o2, l2, rows)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs,n", [(28, 4, 128, 16, 1171), (4, 2, 64, 32, 4097), (32, 8, 128, 64, 2049), (8, 1, 64, 16, 1025)])
def test_long_chunks(fmt, hq, hkv, d, bs, n):
    """A chunk of more than 8192 rows a kv head, whose blocks are staged, beside a
    middle one, a short one and a decode; alone; and on a long prefix."""
    ctx, ql = [n + 77, 150, 40, 500], [n, 100, 2, 1]
    c = Cache(ctx, hq, hkv, d, bs, fmt, seed=n)
    c.fill(c.ctx)
    rows = set(c.rng.permutation(sum(ql))[:20].tolist()) | {0, n - 1, n, n + 99, n + 100, n + 101, n + 102}
    plan, *_ = _attend(c, ql, tokens=rows)
    info = plan.info()
    assert info["prefill_items"] > 0 and info["decode_items"] > 0
    one = Cache([n + 900], hq, hkv, d, bs, fmt, seed=n + 1)
    one.fill(one.ctx)
    plan, *_ = _attend(one, [n], tokens={0, 1, n // 2, n - 2, n - 1})
    assert plan.info()["prefill_items"] > 0 and plan.info()["decode_items"] == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,q", [(8, 1, 64, 250), (4, 2, 64, 700), (28, 4, 128, 60), (40, 1, 128, 33)])
def test_middle_chunks_directly(fmt, hq, hkv, d, q):
    """Chunks of hundreds of rows a kv head over the codes: every row, with and
    without a prefix (early rows see a part of a group's ranges only)."""
    ctx = [q + 50, q, q + 333]
    c = Cache(ctx, hq, hkv, d, 16, fmt, seed=q)
    c.fill(c.ctx)
    rows = set(c.rng.permutation(3 * q)[:60].tolist()) | {0, q - 1, q, q + 1, q + 15, q + 16, q + 17, 2 * q - 1, 2 * q, 3 * q - 1}
    plan, *_ = _attend(c, [q, q, q], tokens=rows)
    assert plan.info()["prefill_items"] == 0
    _attend(c, [q, q, q], tokens=rows, opts=c.fnpu.PlanOpts(48, 0, 0, 0))


@pytest.mark.parametrize("fmt", FMTS)
def test_step_replan_stream_capture(fmt):
    """fnpu_mixed_step stores and attends; the plan is re-planned for the next step;
    runs on another stream and replayed from a graph give the same bits."""
    import paper_2606_04415_gb300 as fnpu
    ctx, ql = np.array([100, 17, 257], np.int32), np.array([90, 1, 1], np.int32)
    c = Cache(ctx + 1, 8, 4, 64, 16, fmt, seed=31)
    c.ctx = ctx
    c.fill(ctx - ql)
    plan = fnpu.kv8_attn_plan(c.desc, fmt, ql, ctx, (ql == 1).astype(np.uint8), c.table)
    for step in range(2):
        T = int(ql.sum())
        sl = np.concatenate([c.slots(s, int(x - n), int(x)) for s, (x, n) in enumerate(zip(ctx, ql))])
        k, v, q = c.rows(T), c.rows(T), _bf16(c.rng, T, 8, 64).cuda()
        out, lse = torch.empty((T, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((T, 8), device="cuda")
        fnpu.mixed_step(plan, k.cuda(), v.cuda(), torch.from_numpy(sl).cuda(), q, *c.dev, out, lse)
        assert fnpu.plan_check(plan) == fnpu.FNPU_OK and fnpu.check() == fnpu.FNPU_OK
        for pool, x in zip(c.pools, (k, v)):
            K8.append(pool, x.double().numpy(), sl, 4, 16, 64, fmt)
        c.same()
        c.ctx = ctx
        _compare(c, ql, q, out, lse)
        if step == 0:
            ctx, ql = ctx + 1, np.ones(3, np.int32)
            fnpu.mixed_attn_replan(plan, ql, ctx, np.ones(3, np.uint8), c.table)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        fnpu.mixed_attn_run(plan, q, *c.dev, o2, l2)
    s.synchronize()
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    g = torch.cuda.CUDAGraph()
    o2.zero_()
    with torch.cuda.graph(g):
        fnpu.mixed_attn_run(plan, q, *c.dev, o2, l2)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o2, out) and torch.equal(l2, lse)


def test_large_pool_offsets():
    """Blocks past 2^32 bytes of a pool."""
    import paper_2606_04415_gb300 as fnpu
    hq, hkv, d, bs, fmt = 16, 8, 128, 64, K8.INT8
    b = K8.block_bytes(hkv, bs, d)
    blocks = (1 << 32) // b + 40
    if torch.cuda.mem_get_info()[0] < 3 * blocks * b:
        pytest.skip("needs 13 GB of device memory")
    rng = np.random.default_rng(41)
    ids = np.array([[blocks - 1, 5, blocks - 20, 2, blocks - 7]], np.int32)
    ctx = 5 * bs - 9
    pos = np.arange(ctx)
    sl = ids[0, pos // bs].astype(np.int64) * bs + pos % bs
    desc = fnpu.make_desc(hq, hkv, d, d, bs, blocks)
    dev = [torch.zeros(blocks * b, dtype=torch.uint8, device="cuda") for _ in range(2)]
    k, v = (_bf16(rng, ctx, hkv, d).cuda() for _ in range(2))
    fnpu.rope_append(desc, None, None, None, None, k, v, torch.from_numpy(sl).cuda(), None, *dev, kv_format=fmt)
    out = [torch.empty((ctx, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    fnpu.kv_read(desc, torch.from_numpy(sl).cuda(), *dev, *out, kv_format=fmt)
    small = np.arange(ctx, dtype=np.int64)
    pools = [np.zeros(5 * b, np.uint8) for _ in range(2)]
    for pool, x, o in zip(pools, (k, v), out):
        K8.append(pool, x.double().cpu().numpy(), small, hkv, bs, d, fmt)
        assert np.array_equal(o.double().cpu().numpy(), K8.read(pool, small, hkv, bs, d, fmt))
    for ql in (1, 60):
        q = _bf16(rng, ql, hq, d).cuda()
        o, l = torch.empty((ql, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((ql, hq), device="cuda")
        plan = fnpu.kv8_attn_plan(desc, fmt, [ql], [ctx], [int(ql == 1)], ids)
        fnpu.mixed_attn_run(plan, q, *dev, o, l)
        assert fnpu.plan_check(plan) == fnpu.FNPU_OK
        ref_o, ref_l = K8.attention(q.double().cpu().numpy(), [ql], [ctx], np.arange(5)[None], *pools, hkv, bs, d, fmt)
        tol = 2.0 ** -8 * np.abs(ref_o) + (2.0 ** -10 if ql == 1 else 2.0 ** -7) * 6
        assert (np.abs(o.double().cpu().numpy() - ref_o) <= tol).all()
        assert (np.abs(l.double().cpu().numpy() - ref_l) <= 2e-5 * np.maximum(1, np.abs(ref_l))).all()
    assert fnpu.check() == fnpu.FNPU_OK


@pytest.mark.parametrize("seed", range(24))
def test_random_steps(seed):
    """Steps of a random layout, batch and mix of lengths, with the planner's own rows
    and ranges: of one-token decodes (even seeds), or with several tokens and chunks."""
    r = np.random.default_rng(1000 + seed)
    hq, hkv, d, bs = LAYOUTS[r.integers(len(LAYOUTS))]
    n = int(np.exp(r.uniform(0, np.log(60))))
    ctx = np.exp(r.uniform(0, np.log([300, 3000, 20000][r.integers(3)] if n < 12 else 1500), n)).astype(int)
    ql = np.ones(n, int) if seed % 2 == 0 else np.minimum(ctx, r.choice([1, 1, 2, 3, 5, 9, 40, 130], n))
    c = Cache(ctx.tolist(), hq, hkv, d, bs, FMTS[r.integers(2)], seed=seed)
    c.fill(c.ctx)
    ends = np.cumsum(ql)
    rows = set(r.permutation(int(ends[-1]))[:40].tolist()) | set((ends - 1)[:12].tolist()) | set((ends - ql)[:12].tolist())
    _attend(c, ql.tolist(), tokens=rows)
