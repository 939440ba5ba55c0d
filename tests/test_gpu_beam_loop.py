"""The page operations, the appends, the windowed attention and the beam selection
together, as a beam search uses them, against rows that keep their whole history."""
import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


class Search:
    """A search whose queries, keys, values and logits are random: ``step`` makes one
    on the device, ``follow`` repeats its choices on rows that own their history."""

    G, W, V, LAYERS = 2, 3, 500, 2

    def __init__(self, heads, bs, window, sinks, prompts, most, seed, blocks=200):
        import paper_2606_04415_gb300 as fnpu
        from paper_2606_04415_gb300.beams import BeamCache
        self.fnpu, self.heads, self.window, self.sinks = fnpu, heads, window or 1 << 30, sinks
        hq, hkv, d = heads
        self.rows = self.G * self.W
        self.cache = BeamCache(hq, hkv, d, bs, blocks, self.LAYERS, self.rows, most, window, sinks)
        for pool in self.cache.k + self.cache.v:
            pool.fill_(float("nan"))               # nothing that was not stored may count
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.lens = [prompts[r // self.W] if r % self.W == 0 else 0 for r in range(self.rows)]
        self.plan, self.slots = self.cache.admit(self.lens)
        self.space = torch.empty(fnpu.beam_select_workspace(self.G, self.W, self.V, self.W), dtype=torch.uint8, device="cuda")
        self.scores = torch.full((self.G, self.W), -float("inf"), device="cuda")
        self.scores[:, 0] = 0
        self.logits = torch.empty((self.G, self.W, self.V), device="cuda")
        self.chosen = [torch.empty((self.G, self.W), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
        self.q, self.k, self.v = ([torch.empty((self.rows, h, d), dtype=torch.bfloat16, device="cuda") for _ in range(self.LAYERS)]
                                  for h in (hq, hkv, hkv))
        self.out, self.lse = ([torch.empty((self.rows, hq, *e), dtype=t, device="cuda") for _ in range(self.LAYERS)]
                              for e, t in (((d,), torch.bfloat16), ((), torch.float32)))
        self.history = [[([], []) for _ in range(self.LAYERS)] for _ in range(self.rows)]

    def normal(self, x, std=1.0):
        x.copy_(torch.randn(x.shape, device="cuda", generator=self.gen) * std)

    def prefill(self):
        hq, hkv, d = self.heads
        n = sum(self.lens)
        got = []
        for layer in range(self.LAYERS):
            q, k, v = (torch.empty((n, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
            for x in (q, k, v):
                self.normal(x)
            got.append((q, *self.cache.prefill(self.plan, self.slots, layer, q, k, v)))
            at = 0
            for r, m in enumerate(self.lens):
                self.history[r][layer] = (list(k[at:at + m].float().cpu().numpy()), list(v[at:at + m].float().cpu().numpy()))
                at += m
        for layer, (q, out, lse) in enumerate(got):
            at = 0
            for r, m in enumerate(self.lens):
                if m:
                    self.check_row(r, layer, q[at:at + m], out[at:at + m], lse[at:at + m], 0)
                at += m

    def inputs(self):
        self.normal(self.logits, 3.0)
        for x in self.q + self.k + self.v:
            self.normal(x)

    def step(self):
        self.fnpu.beam_select(self.logits, self.scores, *self.chosen, self.space)
        self.scores.copy_(self.chosen[0])
        self.cache.advance(self.chosen[1].view(-1))
        for layer in range(self.LAYERS):
            out, lse = self.cache.attend(layer, self.q[layer], self.k[layer], self.v[layer])
            self.out[layer].copy_(out)
            self.lse[layer].copy_(lse)

    def check_row(self, r, layer, q, out, lse, first):
        from oracle import window as O
        k, v = (np.stack(x)[None] for x in self.history[r][layer])
        ref = O.attend(q.float().cpu().numpy(), k, v, [0], first, k.shape[1], self.window, self.sinks)
        to_out, to_lse = O.bounds(*ref, q.shape[2])
        assert (np.abs(out.float().cpu().numpy() - ref[0]) <= to_out).all(), (r, layer)
        assert (np.abs(lse.cpu().numpy() - ref[1]) <= to_lse).all(), (r, layer)

    def follow(self, scores_before):
        from oracle import pages as P
        ref = P.beam_select(self.logits.cpu().numpy(), scores_before.cpu().numpy(), None, self.W, -1)
        parents = self.chosen[1].view(-1).tolist()
        assert np.array_equal(self.chosen[1].cpu().numpy(), ref[1]) and np.array_equal(self.chosen[2].cpu().numpy(), ref[2])
        self.history = [[(list(k), list(v)) for k, v in self.history[p]] for p in parents]
        for r in range(self.rows):
            for layer in range(self.LAYERS):
                for x, new in zip(self.history[r][layer], (self.k, self.v)):
                    x.append(new[layer][r].float().cpu().numpy())
        assert self.cache.length.tolist() == [len(self.history[r][0][0]) for r in range(self.rows)]
        for r in range(self.rows):
            for layer in range(self.LAYERS):
                n = len(self.history[r][layer][0])
                self.check_row(r, layer, self.q[layer][r:r + 1], self.out[layer][r:r + 1], self.lse[layer][r:r + 1], n - 1)
        # every page has as many holders as the table says
        table, n, bs = self.cache.table.cpu().numpy(), self.cache.length.cpu().numpy(), self.cache.block_size
        held = np.concatenate([table[r, :-(-n[r] // bs)] for r in range(self.rows)])
        assert np.array_equal(np.bincount(held[held >= 0], minlength=len(self.cache.refs)), self.cache.refs.cpu().numpy())


CASES = [((28, 4, 128), 16, 40, 3, (70, 33)), ((4, 2, 64), 32, None, 0, (64, 1)), ((16, 8, 128), 16, 17, 0, (5, 100)), ((6, 6, 64), 64, 1, 20, (30, 31))]


@pytest.mark.parametrize("heads,bs,window,sinks,prompts", CASES)
def test_search(heads, bs, window, sinks, prompts):
    s = Search(heads, bs, window, sinks, prompts, 130, seed=bs + sum(heads))
    s.prefill()
    for t in range(20):
        s.inputs()
        before = s.scores.clone()
        s.step()
        s.follow(before)
        if t == 11:
            live = int((s.cache.refs > 0).sum())
            s.cache.compact()
            assert s.cache.moved[0].item() == live and s.cache.refs[:live].gt(0).all() and s.cache.refs[live:].eq(0).all()
    assert s.fnpu.check() == 0 and s.fnpu.plan_check(s.plan) == 0 and s.cache.stats[2].item() == 0
    ends = torch.ones(s.rows, dtype=torch.uint8, device="cuda")
    s.cache.end(ends)
    assert s.cache.refs.eq(0).all() and s.cache.length.eq(0).all()


def test_captured_search():
    """Two steps in a graph, replayed on other inputs: what the history gives."""
    s = Search((28, 4, 128), 16, 40, 3, (70, 33), 130, seed=3)
    s.prefill()
    for _ in range(2):
        s.inputs()
        before = s.scores.clone()
        s.step()
        s.follow(before)
    # the inputs of a captured pair of steps: the second's come from a second buffer
    graph, second = torch.cuda.CUDAGraph(), [torch.empty_like(x) for x in (s.logits, *s.q, *s.k, *s.v)]
    kept = [torch.empty_like(x) for x in (*s.chosen, *s.out, *s.lse, s.cache.tables[0], s.cache.lengths[0], s.cache.refs)]
    now = s.cache.now
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.step()
        for x, y in zip(kept, (*s.chosen, *s.out, *s.lse, s.cache.table, s.cache.length, s.cache.refs)):
            x.copy_(y)
        for x, y in zip((s.logits, *s.q, *s.k, *s.v), second):
            x.copy_(y)
        s.step()
    assert s.cache.now == now
    for _ in range(6):
        s.inputs()
        first = [x.clone() for x in (s.logits, *s.q, *s.k, *s.v)]
        s.inputs()
        for x, y, z in zip((s.logits, *s.q, *s.k, *s.v), second, first):
            y.copy_(x)
            x.copy_(z)
        before = s.scores.clone()
        graph.replay()
        torch.cuda.synchronize()
        after = [x.clone() for x in (*s.chosen, *s.out, *s.lse, s.cache.table, s.cache.length, s.cache.refs)]
        state = (*s.chosen, *s.out, *s.lse, s.cache.table, s.cache.length, s.cache.refs)
        last, held = [x.clone() for x in (s.logits, *s.q, *s.k, *s.v)], s.scores.clone()
        # the first of the two steps, then the second
        for x, y in zip(state, kept):
            x.copy_(y)
        for x, y in zip((s.logits, *s.q, *s.k, *s.v), first):
            x.copy_(y)
        s.follow(before)
        before = s.chosen[0].clone()
        for x, y in zip((*state, s.logits, *s.q, *s.k, *s.v), (*after, *last)):
            x.copy_(y)
        s.follow(before)
        assert torch.equal(s.scores, held)
    assert s.fnpu.check() == 0


def test_rows_without_a_free_block():
    """A pool that runs out: the rows that find no block stay as they were, the others go on."""
    s = Search((4, 2, 64), 16, None, 0, (32, 32), 130, seed=9, blocks=5)
    s.prefill()                                    # 2 blocks each, one is free
    s.inputs()
    s.step()                                       # six rows want a block of their own
    assert s.cache.stats.tolist() == [0, 1, 5, 0]
    assert s.cache.length.tolist() == [33, 32, 32, 32, 32, 32] and s.cache.slots.view(-1)[1:].eq(-1).all()
    for layer in range(s.LAYERS):
        assert torch.isfinite(s.out[layer].float()).all() and torch.isfinite(s.lse[layer]).all()
    assert s.fnpu.check() == 0


def test_admit_refuses():
    from paper_2606_04415_gb300.beams import BeamCache
    c = BeamCache(4, 2, 64, 16, 4, 1, 3, 40)
    for bad in ([1, 2], [1, 2, -1], [41, 0, 0], [33, 33, 0]):
        with pytest.raises(ValueError):
            c.admit(bad)


def _loop():
    spec = importlib.util.spec_from_file_location("beam_search_loop", os.path.join(ROOT, "examples", "beam_search_loop.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_captured_and_eager_agree():
    args = ["--heads", "8", "2", "64", "--requests", "2", "--beams", "3", "--prompt", "90", "--tokens", "12", "--window", "40", "--vocab", "2003"]
    got = [_loop().main(args + extra) for extra in ([], ["--eager"])]
    assert np.array_equal(got[0]["text"], got[1]["text"]) and np.array_equal(got[0]["scores"], got[1]["scores"])
    assert got[0]["unserved"] == 0 and (np.diff(got[0]["scores"], axis=1) <= 0).all()
