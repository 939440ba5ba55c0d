"""Attention with a sliding window and sinks against the fp64 reference.

Every row is held to a bound by its own weights (oracle.window.bounds): one
rounding of each weight and of the output to bf16, fp32 scores and sums. Blocks
that no query sees are gone from the table (ids that no pool has, or other
sequences'), and hidden rows of the blocks that are there hold NaN and infinities."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HUGE = 2 ** 31 - 1


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def _needed(c, q, bs, window, sinks):
    from oracle.window import visible
    seen = set()
    for p in range(c - q, c):
        seen |= set(visible(p, window, sinks))
    return seen


class Step:
    """A step's tensors; ``junk``: what entries of blocks that are gone hold."""

    def __init__(self, heads, bs, seqs, window, sinks, seed=0, junk=-1, poison=True):
        self.heads, self.bs, self.window, self.sinks = heads, bs, window, sinks
        hq, hkv, d = heads
        rng = np.random.default_rng([41, seed])
        self.q_len, self.ctx, self.phase = (np.array(a, t) for a, t in zip(zip(*seqs), (np.int32, np.int32, np.uint8)))
        seen = [_needed(int(c), int(q), bs, window, sinks) for q, c in zip(self.q_len, self.ctx)]
        cols = [sorted({j // bs for j in s}) for s in seen]
        self.blocks = sum(map(len, cols)) + 3
        perm, at = rng.permutation(self.blocks), 0
        self.table = np.full((len(seqs), int(-(-self.ctx.max() // bs)) + 1), junk, np.int32)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = (torch.randn((self.blocks, bs, hkv, d), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
        self.q = (2 * torch.randn((int(self.q_len.sum()), hq, d), device="cuda", generator=g)).to(torch.bfloat16)
        live = np.zeros((self.blocks, bs), bool)
        for s, c in enumerate(cols):
            self.table[s, c] = perm[at:at + len(c)]
            at += len(c)
            j = np.array(sorted(seen[s]))
            live[self.table[s, j // bs], j % bs] = True
        if poison:
            dead = torch.from_numpy(~live).cuda()
            self.k[dead], self.v[dead] = float("nan"), float("inf")
        self.out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full(self.q.shape[:2], 7.0, device="cuda")
        import paper_2606_04415_gb300 as fnpu
        self.fnpu = fnpu
        self.desc = fnpu.make_desc(hq, hkv, d, d, bs, self.blocks)

    def plan(self, opts=None):
        return self.fnpu.window_attn_plan(self.desc, self.window, self.sinks, self.q_len, self.ctx, self.phase, self.table, opts=opts)

    def run(self, plan):
        self.fnpu.mixed_attn_run(plan, self.q, self.k, self.v, self.out, self.lse)
        torch.cuda.synchronize()
        assert self.fnpu.plan_check(plan) == 0 and self.fnpu.check() == 0

    def device(self):
        return torch.from_numpy(self.ctx).cuda(), torch.from_numpy(self.table).cuda()

    def workspace(self, most=None, split=0):
        n = self.fnpu.window_decode_workspace(self.desc, self.window, self.sinks, len(self.ctx), most or int(self.ctx.max()), split)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")

    def check(self, rows=None):
        """Rows of the sequences ``rows`` (all by default) within their bounds."""
        from oracle import window as W
        q, k, v = (x.float().cpu().numpy() for x in (self.q, self.k, self.v))
        out, lse = self.out.float().cpu().numpy(), self.lse.cpu().numpy()
        at = 0
        for s, (n, c) in enumerate(zip(self.q_len, self.ctx)):
            if rows is None or s in rows:
                ref = W.attend(q[at:at + n], k, v, self.table[s], int(c - n), self.bs, self.window, self.sinks)
                to_out, to_lse = W.bounds(*ref, q.shape[2])
                assert np.isfinite(out[at:at + n]).all(), f"sequence {s}"
                bad = np.abs(out[at:at + n] - ref[0]) / to_out
                off = np.abs(lse[at:at + n] - ref[1]) / to_lse
                assert bad.max() <= 1 and off.max() <= 1, f"sequence {s}: {bad.max()} {off.max()} at row {np.unravel_index(bad.argmax(), bad.shape)}"
            at += n


HEADS = [(4, 2, 64), (8, 1, 64), (6, 6, 128), (28, 4, 128), (16, 5 - 1, 64), (24, 6, 128), (32, 8, 128)]
WINDOWS = [(1, 0), (1, 3), (5, 4), (16, 0), (17, 16), (100, 17), (128, 1), (129, 130), (300, 40), (1000, 0), (HUGE, 0), (HUGE, HUGE), (3, HUGE)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("heads,bs", [((28, 4, 128), 16), ((4, 2, 64), 64), ((24, 6, 128), 48)])
def test_decodes(heads, bs, window, sinks):
    ctx = [1, 2, 15, 16, 17, 33, 100, 129, 144, 400, 777] + [c for c in (window, window + 1, window + sinks + 16) if c < 1500]
    st = Step(heads, bs, [(1, c, 1) for c in ctx], window, sinks, seed=window % 1000 + sinks % 1000)
    st.run(st.plan())
    st.check()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("bs,window,sinks", [(16, 100, 4), (32, 37, 40)])
def test_chunks(heads, bs, window, sinks):
    st = Step(heads, bs, [(150, 150, 0), (67, 500, 0), (1, 300, 0), (5, 333, 1)], window, sinks, seed=7, junk=2 ** 30)
    st.run(st.plan())
    st.check()


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("heads,bs", [((28, 4, 128), 64), ((8, 1, 64), 16)])
def test_chunk_windows(heads, bs, window, sinks):
    st = Step(heads, bs, [(40, 300, 0), (131, 131, 0), (3, 400, 1), (20, 20, 0)], window, sinks, seed=9)
    st.run(st.plan())
    st.check()


@pytest.mark.parametrize("window,sinks", [(60, 4), (700, 0), (128, 300)])
def test_mixed(window, sinks):
    st = Step((28, 4, 128), 16, [(200, 900, 0), (1, 700, 1), (1, 1, 1), (90, 90, 0), (1, 333, 1), (4, 600, 1)], window, sinks, seed=11)
    st.run(st.plan())
    st.check()
    for flags in (st.fnpu.PLAN_SEPARATE_LAUNCHES, st.fnpu.PLAN_GREEN_CONTEXTS):
        first = st.out.clone()
        st.out.fill_(7.0)
        st.run(st.plan(st.fnpu.PlanOpts(0, 0, 0, flags)))
        st.check()
        assert first.shape == st.out.shape


@pytest.mark.parametrize("flags,share", [(1, 0), (4, 0), (4, 40), (0, 10)])
def test_mixed_in_every_way_of_running(flags, share):
    """Both phases in launches of their own, in green contexts, and with a share that is asked for."""
    import paper_2606_04415_gb300 as fnpu
    st = Step((16, 8, 64), 32, [(90, 700, 0), (33, 33, 0), (200, 201, 0)] + [(1, c, 1) for c in (1, 40, 300, 777, 2000)], 130, 20, seed=flags + share)
    st.run(st.plan(fnpu.PlanOpts(0, share, 0, flags)))
    st.check()


@pytest.mark.parametrize("n,ctx,window", [(120, 900, 800), (300, 700, 400)])
def test_more_rows_than_fit_at_once(n, ctx, window):
    """Items of more than a round, planned and not, lengths that vary past the window."""
    rng = np.random.default_rng([53, n])
    st = Step((8, 8, 64), 16, [(1, int(c), 1) for c in rng.integers(ctx, 3 * ctx, n)], window, 5, seed=n)
    st.run(st.plan())
    some = list(range(0, n, 17))
    st.check(some)
    st.out.fill_(7.0), st.lse.fill_(7.0)
    _decode(st, *st.device(), int(st.ctx.max()), st.workspace())
    st.check(some)


@pytest.mark.parametrize("split", [16, 64, 1000])
@pytest.mark.parametrize("window,sinks", [(300, 20), (64, 0)])
def test_decode_splits(split, window, sinks):
    """Every cut of the virtual keys, the gap inside a piece and between two."""
    st = Step((32, 8, 128), 16, [(1, c, 1) for c in (5, 64, 321, 340, 700)], window, sinks, seed=13)
    st.run(st.plan(st.fnpu.PlanOpts(split, 0, 0, 0)))
    st.check()


@pytest.mark.parametrize("window,sinks", [(2300, 0), (1700, 600), (2600, 5)])
@pytest.mark.parametrize("heads", [(8, 8, 64), (28, 4, 128)])
def test_chunk_pieces_that_rows_do_not_see(heads, window, sinks):
    """A few units on many SMs are cut into pieces, some of which lie outside the windows of some rows."""
    st = Step(heads, 16, [(200, 3500, 0)], window, sinks, seed=15)
    plan = st.plan()
    units = (200 + 2 * (128 // (heads[0] // heads[1])) - 1) // (2 * (128 // (heads[0] // heads[1]))) * heads[1]
    assert plan.info()["prefill_items"] > units
    st.run(plan)
    st.check()
    first = st.out.clone()
    st.run(plan)
    assert torch.equal(first, st.out)


def test_replan_keeps_the_window_and_runs_repeat():
    st = Step((28, 4, 128), 16, [(1, 500, 1), (40, 200, 0)], 90, 4, seed=17)
    plan = st.plan()
    st.run(plan)
    st.check()
    st2 = Step((28, 4, 128), 16, [(33, 1000, 0), (1, 800, 1), (1, 30, 1)], 90, 4, seed=18)
    assert st2.blocks != st.blocks    # (a plan is of one pool: the larger one serves both)
    big = st if st.blocks > st2.blocks else st2
    plan = big.plan()
    st2.desc = st.desc = big.desc
    for a in (st, st2):
        pool = [torch.zeros_like(big.k), torch.zeros_like(big.v)]
        for p, x in zip(pool, (a.k, a.v)):
            p[:a.blocks] = x
        a.k, a.v = pool
        st.fnpu.mixed_attn_replan(plan, a.q_len, a.ctx, a.phase, a.table)
        a.run(plan)
        a.check()


@pytest.mark.parametrize("flags", [0, 8])
def test_step_appends_first(flags):
    """fnpu_mixed_step with a window: a step's queries see its own new keys."""
    st = Step((28, 4, 128), 16, [(100, 300, 0), (1, 260, 1), (1, 17, 1)], 64, 4, seed=19)
    hq, hkv, d = st.heads
    new = [torch.randn((102, hkv, d), device="cuda").to(torch.bfloat16) for _ in range(2)]
    pos = np.concatenate([np.arange(c - n, c) for n, c in zip(st.q_len, st.ctx)])
    seq = np.repeat(np.arange(3), st.q_len)
    slots = torch.from_numpy(st.table[seq, pos // 16].astype(np.int64) * 16 + pos % 16).cuda()
    plan = st.plan(st.fnpu.PlanOpts(0, 0, 0, flags))
    st.fnpu.mixed_step(plan, *new, slots, st.q, st.k, st.v, st.out, st.lse)
    torch.cuda.synchronize()
    assert st.fnpu.plan_check(plan) == 0 and st.fnpu.check() == 0
    assert torch.equal(st.k.view(-1, hkv, d)[slots], new[0]) and torch.equal(st.v.view(-1, hkv, d)[slots], new[1])
    st.check()


# ------------------------------------------------------- without a plan

def _decode(st, ctx, table, most, ws, split=0, stream=None):
    st.fnpu.window_decode(st.desc, st.window, st.sinks, ctx, table, most, st.q, st.k, st.v, st.out, st.lse, ws, split_keys=split,
                          stream=stream)


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("heads,bs", [((28, 4, 128), 16), ((4, 2, 64), 64), ((24, 6, 128), 48)])
def test_rows(heads, bs, window, sinks):
    ctx = [1, 2, 15, 16, 17, 33, 100, 129, 144, 400, 777] + [c for c in (window, window + 1, window + sinks + 16) if c < 1500]
    st = Step(heads, bs, [(1, c, 1) for c in ctx], window, sinks, seed=window % 1000 + sinks % 1000, junk=2 ** 30)
    most = st.table.shape[1] * bs
    for split in (0, 64):
        st.out.fill_(7.0)
        _decode(st, *st.device(), most, st.workspace(most, split), split)
        torch.cuda.synchronize()
        assert st.fnpu.check() == 0
        st.check()


def test_rows_without_keys_and_out_of_range():
    st = Step((28, 4, 128), 16, [(1, c, 1) for c in (300, 9, 500, 40, 200)], 100, 4, seed=21)
    ctx, table = st.device()
    ctx[1], ctx[3], ctx[4] = 0, -5, 513
    ref = st.out.clone()
    _decode(st, ctx, table, 512, st.workspace(512))
    torch.cuda.synchronize()
    assert st.fnpu.check() == st.fnpu.FNPU_EDEVICE_RANGE and st.fnpu.check() == 0
    st.check(rows=(0, 2))
    assert (st.out[1] == 0).all() and (st.lse[1] == -float("inf")).all()
    for s in (3, 4):
        assert torch.equal(st.out[s], ref[s]) and (st.lse[s] == 7.0).all()


def test_rows_flag_visible_blocks_out_of_range():
    st = Step((4, 2, 64), 16, [(1, 300, 1), (1, 200, 1), (1, 100, 1)], 50, 4, seed=23)
    ctx, table = st.device()
    table[1, 0], table[2, 5] = st.blocks, -1       # a sink's block, one of a window
    _decode(st, ctx, table, 300, st.workspace(300))
    torch.cuda.synchronize()
    assert st.fnpu.check() == st.fnpu.FNPU_EDEVICE_RANGE
    st.check(rows=(0,))


def test_rows_captured_and_replayed_with_other_lengths():
    """The same graph on later lengths, as a decode loop replays it, and two graphs at once on two workspaces."""
    a, b = (Step((28, 4, 128), 16, [(1, c, 1) for c in ctx], 200, 4, seed=25) for ctx in ((700, 350, 30), (201, 999, 640)))
    most = 1024
    state = []
    for st in (a, b):
        ctx, table = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.full((3, 64), -1, dtype=torch.int32, device="cuda")
        ws, s, g = st.workspace(most), torch.cuda.Stream(), torch.cuda.CUDAGraph()
        _decode(st, ctx, table, most, ws)
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            _decode(st, ctx, table, most, ws)
        state.append((st, ctx, table, ws, s, g))
    for _ in range(3):
        for st, ctx, table, ws, s, g in state:
            st.out.fill_(7.0)
            ctx.copy_(torch.from_numpy(st.ctx))
            table[:, :st.table.shape[1]] = torch.from_numpy(st.table).cuda()
        torch.cuda.synchronize()
        for st, ctx, table, ws, s, g in state:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for st, *_ in state:
            st.check()
    assert a.fnpu.check() == 0


def test_rows_binding_checks():
    st = Step((4, 2, 64), 16, [(1, 30, 1), (1, 20, 1)], 10, 2, seed=27)
    ctx, table = st.device()
    ws = st.workspace(32)
    for bad in (dict(ctx=ctx.long()), dict(table=table[:1]), dict(table=table.long()), dict(table=table.t().contiguous().t())):
        with pytest.raises((TypeError, ValueError)):
            _decode(st, bad.get("ctx", ctx), bad.get("table", table), 32, ws)
    st.out = st.out.float()
    with pytest.raises(ValueError):
        _decode(st, ctx, table, 32, ws)
