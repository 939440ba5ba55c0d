"""The page operations on the device against the row-by-row reference: equal in every value."""
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


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype))).cuda()


class State:
    """A random state: rows that share prefixes, some pages held elsewhere too."""

    def __init__(self, seed, rows, width, bs, blocks, most=None, freed=0.0, outside=0.05):
        from oracle import pages as P
        rng = np.random.default_rng([43, seed])
        self.rng, self.bs, self.width, self.blocks = rng, bs, width, blocks
        most = width * bs if most is None else most
        self.n = rng.integers(0, most + 1, rows)
        perm, at = rng.permutation(blocks), 0
        self.rows = []
        for r in range(rows):
            k = P.held(int(self.n[r]), bs)
            shared = int(rng.integers(0, min(k, len(self.rows[-1])) + 1)) if r and rng.random() < 0.7 else 0
            row = list(self.rows[-1][:shared]) if shared else []
            fresh = k - len(row)
            assert at + fresh <= blocks
            row += [int(e) for e in perm[at:at + fresh]]
            at += fresh
            self.rows.append([-1 if c + 1 < k and rng.random() < freed else e for c, e in enumerate(row)])
        self.refs = np.bincount([e for row in self.rows for e in row if e >= 0], minlength=blocks)
        extra = rng.random(blocks) < outside
        self.refs[extra & (self.refs > 0)] += 1
        import paper_2606_04415_gb300 as fnpu
        self.fnpu = fnpu
        self.desc = fnpu.make_pages(bs, blocks)

    def table(self, rows=None, junk=None):
        """Entries past a row's pages: anything."""
        rows = self.rows if rows is None else rows
        t = self.rng.integers(-5, self.blocks + 5, (len(rows), self.width)) if junk is None else np.full((len(rows), self.width), junk)
        for r, row in enumerate(rows):
            t[r, :len(row)] = row
        return _dev(t, np.int32)

    def workspace(self, rows):
        n = self.fnpu.pages_workspace(self.desc, rows)
        return torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda")   # nothing is kept in it


def _outputs(st, new, grow):
    e = lambda *s, t=torch.int32: torch.full(s, 77, dtype=t, device="cuda")  # noqa: E731
    return e(new, st.width), e(new), e(new, grow, t=torch.int64), e(new, 2), e(4)


def _check_fork(st, parents, grow, got, refs):
    from oracle import pages as P
    rows, n, want_refs, slots, copies, stats = P.fork(st.rows, st.n, st.refs, st.bs, st.width, parents, grow)
    assert got[4].tolist() == stats
    assert got[1].tolist() == n
    assert got[0].tolist() == [r + [-1] * (st.width - len(r)) for r in rows]
    assert refs.tolist() == [int(c) for c in want_refs]
    assert got[3].tolist() == copies
    assert got[2].tolist() == slots


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("rows,new,width,bs,blocks,grow", [(4, 4, 9, 16, 60, 1), (1, 8, 3, 4, 5, 2), (9, 3, 20, 1, 200, 5), (8, 8, 130, 64, 1100, 1),
                                                           (3, 12, 7, 32, 40, 100), (600, 700, 5, 16, 20000, 1), (5, 5, 6, 16, 40, 0),
                                                           (2, 5000, 4, 16, 9000, 1)])
def test_fork(seed, rows, new, width, bs, blocks, grow):
    st = State(seed, rows, width, bs, blocks, most=max(1, width * bs - (grow if seed % 2 else 0)))
    parents = st.rng.integers(-1 if seed % 3 else 0, rows, new)
    refs, got = _dev(st.refs, np.int32), _outputs(st, new, grow)
    st.fnpu.pages_fork(st.desc, st.table(), _dev(st.n, np.int32), refs, *got, st.workspace(max(rows, new)), parents=_dev(parents, np.int32))
    torch.cuda.synchronize()
    assert st.fnpu.check() in (0, st.fnpu.FNPU_EDEVICE_RANGE) and st.fnpu.check() == 0
    _check_fork(st, parents.tolist(), grow, got, refs)


@pytest.mark.parametrize("seed", range(3))
def test_fork_raises_no_flag_on_a_sound_state(seed):
    st = State(seed, 20, 12, 16, 400)
    parents = st.rng.integers(0, 20, 24)
    refs, got = _dev(st.refs, np.int32), _outputs(st, 24, 1)
    st.fnpu.pages_fork(st.desc, st.table(), _dev(st.n, np.int32), refs, *got, st.workspace(24), parents=_dev(parents, np.int32))
    assert st.fnpu.check() == 0


@pytest.mark.parametrize("in_place", [False, True])
def test_fork_of_the_same_rows(in_place):
    """Without parents: the rows go on, shared last pages are copied."""
    st = State(5, 30, 10, 16, 400, most=150)
    refs, got, table, n = _dev(st.refs, np.int32), list(_outputs(st, 30, 3)), st.table(), _dev(st.n, np.int32)
    if in_place:
        got[0], got[1] = table, n
    st.fnpu.pages_fork(st.desc, table, n, refs, *got, st.workspace(30))
    torch.cuda.synchronize()
    _check_fork(st, list(range(30)), 3, got, refs)


def test_fork_with_a_tail_that_was_freed_and_bad_parents():
    st = State(7, 6, 8, 16, 100, most=100)
    st.n[:] = [20, 33, 16, 40, 7, 0]
    at = iter(range(100))
    st.rows = [[next(at) for _ in range(-(-int(n) // 16))] for n in st.n]
    st.rows[0][0], st.rows[1][2] = -1, -1      # a page behind a window; a last page
    st.refs = np.bincount([e for r in st.rows for e in r if e >= 0], minlength=100)
    refs, got = _dev(st.refs, np.int32), _outputs(st, 5, 1)
    parents = [0, 1, 1, 3, 5]
    st.fnpu.pages_fork(st.desc, st.table(junk=-1), _dev(st.n, np.int32), refs, *got, st.workspace(8), parents=_dev(parents, np.int32))
    torch.cuda.synchronize()
    assert st.fnpu.check() == 0
    _check_fork(st, parents, 1, got, refs)
    # a parent past the rows and lengths that no row can have: empty rows, flagged
    refs, got = _dev(st.refs, np.int32), _outputs(st, 4, 1)
    n = _dev([20, 33, 16, 40, 7, 129], np.int32)
    st.fnpu.pages_fork(st.desc, st.table(junk=-1), n, refs, *got, st.workspace(8), parents=_dev([6, 2, 5, 0], np.int32))
    assert st.fnpu.check() == st.fnpu.FNPU_EDEVICE_RANGE
    assert got[1].tolist() == [0, 17, 0, 21] and got[2][0].item() == got[2][2].item() == -1
    # an id past the pool: flagged, and a freed entry from then on
    refs, got, t = _dev(st.refs, np.int32), _outputs(st, 1, 1), st.table(junk=-1)
    t[3, 0] = 100
    st.fnpu.pages_fork(st.desc, t, _dev(st.n, np.int32), refs, *got, st.workspace(8), parents=_dev([3], np.int32))
    assert st.fnpu.check() == st.fnpu.FNPU_EDEVICE_RANGE and got[0][0, 0].item() == -1


def test_fork_of_no_rows():
    st = State(8, 3, 4, 16, 20)
    refs, got = _dev(st.refs, np.int32), _outputs(st, 0, 1)
    st.fnpu.pages_fork(st.desc, st.table(junk=-1), _dev(st.n, np.int32), refs, *got, st.workspace(3), parents=_dev([], np.int32))
    torch.cuda.synchronize()
    _check_fork(st, [], 1, got, refs)
    st = State(9, 0, 4, 16, 20)
    refs, got = _dev(st.refs, np.int32), _outputs(st, 2, 1)
    st.fnpu.pages_fork(st.desc, st.table(junk=-1), _dev(st.n, np.int32), refs, *got, st.workspace(3), parents=_dev([-1, -1], np.int32))
    torch.cuda.synchronize()
    assert got[4].tolist() == [20, 0, 0, 0] and got[0].eq(-1).all()


@pytest.mark.parametrize("window,sinks,ends", [(0, 0, True), (1, 0, False), (5, 3, True), (16, 16, True), (40, 1, False), (47, 17, True),
                                               (2 ** 31 - 1, 4, True), (3, 2 ** 31 - 1, False)])
@pytest.mark.parametrize("rows,width,bs,blocks", [(7, 9, 16, 100), (40, 300, 1, 12000), (5, 4, 64, 30)])
def test_free(rows, width, bs, blocks, window, sinks, ends):
    from oracle import pages as P
    st = State(window % 100 + rows, rows, width, bs, blocks, freed=0.2)
    flags = (st.rng.random(rows) < 0.3).astype(np.uint8) if ends else None
    refs, n, table = _dev(st.refs, np.int32), _dev(st.n, np.int32), st.table()
    before = table.clone()
    st.fnpu.pages_free(st.desc, table, n, refs, ends=None if flags is None else _dev(flags, np.uint8), window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert st.fnpu.check() == 0
    want, lens, counts = P.free(st.rows, st.n, st.refs, bs, flags, window, sinks)
    assert refs.tolist() == [int(c) for c in counts] and n.tolist() == lens
    for r, row in enumerate(want):
        assert table[r, :len(row)].tolist() == row
        assert torch.equal(table[r, len(row):], before[r, len(row):])


def test_free_flags_counts_that_are_not_there():
    st = State(11, 3, 4, 16, 20)
    table, n, refs = _dev([[1, 2, -1, -1], [3, 25, -1, -1], [0, 0, 0, 0]], np.int32), _dev([30, 20, 65], np.int32), torch.zeros(20, dtype=torch.int32, device="cuda")
    refs[1] = 1
    st.fnpu.pages_free(st.desc, table, n, refs, ends=torch.ones(3, dtype=torch.uint8, device="cuda"))
    assert st.fnpu.check() == st.fnpu.FNPU_EDEVICE_RANGE
    assert refs.eq(0).all() and n.tolist() == [0, 0, 65] and table[:2].eq(-1).all() and table[2].eq(0).all()


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("rows,width,bs,blocks,most", [(5, 8, 16, 60, 100), (30, 40, 16, 3000, 3000), (600, 20, 4, 30000, 30000), (4, 6, 16, 90, 3),
                                                       (3, 5, 16, 15, 9), (0, 4, 16, 9000, 5), (2, 4, 16, 8, 0)])
def test_compact(seed, rows, width, bs, blocks, most):
    from oracle import pages as P
    st = State(seed, rows, width, bs, blocks, freed=0.1, outside=0.3)
    if rows and seed == 3:   # pages that only something else holds
        st.refs[st.rng.integers(0, blocks, max(1, blocks // 9))] += 1
    refs, n, table = _dev(st.refs, np.int32), _dev(st.n, np.int32), st.table(junk=-1)
    copies, remap, stats = (torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((most, 2), (blocks,), (2,)))
    st.fnpu.pages_compact(st.desc, table, n, refs, copies, remap, stats, st.workspace(rows))
    torch.cuda.synchronize()
    assert st.fnpu.check() == 0
    want, counts, pairs, where, what = P.compact(st.rows, st.refs, most)
    assert stats.tolist() == what
    assert refs.tolist() == [int(c) for c in counts]
    assert copies.tolist() == pairs + [[-1, -1]] * (most - len(pairs))
    assert remap.tolist() == where
    assert table.tolist() == [r + [-1] * (width - len(r)) for r in want]


def test_compact_of_full_and_empty_pools():
    import paper_2606_04415_gb300 as fnpu
    for refs in (torch.ones(9000, dtype=torch.int32), torch.zeros(9000, dtype=torch.int32)):
        d, r = fnpu.make_pages(16, 9000), refs.cuda()
        copies, remap, stats = (torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((10, 2), (9000,), (2,)))
        t, n = torch.full((1, 3), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        fnpu.pages_compact(d, t, n, r, copies, remap, stats, torch.zeros(fnpu.pages_workspace(d, 1), dtype=torch.uint8, device="cuda"))
        assert stats.tolist() == [int(refs.sum()), 0] and copies.eq(-1).all() and torch.equal(r.cpu(), refs)
        assert remap.tolist() == (list(range(9000)) if refs[0] else [-1] * 9000)


@pytest.mark.parametrize("blocks", [2048, 2049, 2048 * 2048 + 4097])
def test_pools_of_any_size(blocks):
    """Pools of one chunk of counts, of two, and of so many that a chunk is longer."""
    import paper_2606_04415_gb300 as fnpu
    rng = np.random.default_rng([47, blocks])
    refs = (rng.random(blocks) < 0.5).astype(np.int32)
    refs[:100], refs[-50:] = 1, 1
    live, d, rows = np.flatnonzero(refs), fnpu.make_pages(1, blocks), 40
    table = np.full((rows, 600), -1, np.int32)
    table[:, :3] = live[:rows * 3].reshape(rows, 3)
    table[0, 2], table[1, 1] = live[-1], live[-2]
    n, ws = np.full(rows, 3, np.int32), torch.full((fnpu.pages_workspace(d, rows),), 0xFF, dtype=torch.uint8, device="cuda")
    # full pages only: each row takes the next 7 free ids (the pool has some at both ends of every chunk)
    r, got = _dev(refs, np.int32), [torch.full(s, 77, dtype=t, device="cuda") for s, t in
                                    (((rows, 600), torch.int32), ((rows,), torch.int32), ((rows, 7), torch.int64), ((rows, 2), torch.int32), ((4,), torch.int32))]
    fnpu.pages_fork(d, _dev(table, np.int32), _dev(n, np.int32), r, *got, ws)
    free = np.flatnonzero(refs == 0)
    taken = free[:rows * 7].reshape(rows, 7)
    want = refs.copy()
    want[taken] = 1
    assert np.array_equal(got[0].cpu().numpy()[:, 3:10], taken) and np.array_equal(got[2].cpu().numpy(), taken)
    assert got[4].tolist() == [len(free) - rows * 7, rows * 7, 0, 0] and np.array_equal(r.cpu().numpy(), want)
    # compaction: the i-th highest live page to the i-th lowest free place
    refs[live] = rng.integers(1, 9, len(live))
    r, moves = _dev(refs, np.int32), int((live >= len(live)).sum())
    copies, remap, stats = (torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((moves + 3, 2), (blocks,), (2,)))
    t = _dev(table, np.int32)
    fnpu.pages_compact(d, t, _dev(n, np.int32), r, copies, remap, stats, ws)
    src, dst = live[live >= len(live)][::-1], free[free < len(live)]
    where = np.where(refs > 0, np.arange(blocks), -1)
    where[src] = dst
    assert stats.tolist() == [len(live), moves] and np.array_equal(copies.cpu().numpy()[:moves], np.stack([src, dst], 1))
    assert copies[moves:].eq(-1).all() and np.array_equal(remap.cpu().numpy(), where)
    want = np.zeros_like(refs)
    want[where[live]] = refs[live]
    assert np.array_equal(r.cpu().numpy(), want)
    assert np.array_equal(t.cpu().numpy()[:, :3], where[table[:, :3]]) and fnpu.check() == 0


# ---------------------------------------------------------------- copies

def _pools(fnpu, kind, layers, blocks=37):
    if kind == "bf16":
        d, fmt, shape, t = fnpu.make_desc(28, 4, 128, 128, 16, blocks), 0, (blocks, 16, 4, 128), torch.bfloat16
    elif kind == "odd":
        d, fmt, shape, t = fnpu.make_desc(3, 3, 72, 72, 5, blocks), 0, (blocks, 5, 3, 72), torch.bfloat16
    elif kind == "large":
        d, fmt, shape, t = fnpu.make_desc(32, 8, 128, 128, 64, blocks), 0, (blocks, 64, 8, 128), torch.bfloat16
    elif kind == "widths":
        d, fmt, shape, t = fnpu.make_desc(4, 4, 192, 128, 16, blocks), 0, (blocks, 16, 4, 192), torch.bfloat16
    elif kind == "latent":
        d, fmt, shape, t = fnpu.make_desc(64, 1, 576, 512, 64, blocks, latent=True), 0, (blocks, 64, 576), torch.bfloat16
    elif kind == "fp8":
        d, fmt, shape, t = fnpu.make_desc(28, 4, 128, 128, 16, blocks, kv_fp8=True), 0, (blocks, fnpu.FP8_BLOCK_BYTES), torch.uint8
    else:
        d = fnpu.make_desc(6, 3, 64, 64, 32, blocks)
        fmt, t = fnpu.KV_INT8_BLOCK, torch.uint8
        shape = (blocks, fnpu.kv8_block_bytes(d, fmt))
    def make(shape):
        return torch.randint(0, 256, (*shape[:-1], shape[-1] * t.itemsize), dtype=torch.uint8, device="cuda").view(t)
    k = [make(shape) for _ in range(layers)]
    v = None if kind == "latent" else [make((blocks, 16, 4, 128) if kind == "widths" else shape) for _ in range(layers)]
    return d, fmt, k, v


@pytest.mark.parametrize("kind", ["bf16", "odd", "large", "widths", "latent", "fp8", "int8"])
@pytest.mark.parametrize("layers", [1, 3])
def test_copy_blocks(kind, layers):
    import paper_2606_04415_gb300 as fnpu
    d, fmt, k, v = _pools(fnpu, kind, layers)
    pairs = [[3, 9], [-1, -1], [36, 0], [3, 10], [5, -1], [-1, 5], [7, 36 - 1]] + [[-1, -1]] * 50 + [[20, 21]]
    want = [x.view(torch.uint8).reshape(37, -1).clone() for x in k + (v or [])]
    for x in want:
        for s, t in pairs:
            if s >= 0 and t >= 0:
                x[t] = x[s]
    fnpu.kv_copy_blocks(d, _dev(pairs, np.int32), k, v, kv_format=fmt)
    torch.cuda.synchronize()
    assert fnpu.check() == 0
    for x, w in zip(k + (v or []), want):
        assert torch.equal(x.view(torch.uint8).reshape(37, -1), w)


def test_copy_blocks_of_many_layers_and_bad_ids():
    import paper_2606_04415_gb300 as fnpu
    d = fnpu.make_desc(2, 1, 64, 64, 16, 6)
    k, v = ([torch.randn((6, 16, 1, 64), device="cuda").to(torch.bfloat16) for _ in range(130)] for _ in range(2))
    want = [x.clone() for x in k + v]
    for x in want:
        x[4] = x[1]
    fnpu.kv_copy_blocks(d, _dev([[1, 4], [2, 6], [6, 3], [7, -1]], np.int32), k, v)
    assert fnpu.check() == fnpu.FNPU_EDEVICE_RANGE
    assert all(torch.equal(a, b) for a, b in zip(k + v, want))
    with pytest.raises(ValueError):
        fnpu.kv_copy_blocks(d, _dev([[1, 4]], np.int32), k, v[:2])
    with pytest.raises(ValueError):
        fnpu.kv_copy_blocks(d, _dev([[1, 4]], np.int32), [k[0][:5]], [v[0]])
    with pytest.raises(TypeError):
        fnpu.kv_copy_blocks(d, _dev([[1, 4]], np.int64), k, v)


def test_copies_past_32_bits():
    """A pool whose blocks lie past 2^32 bytes."""
    import paper_2606_04415_gb300 as fnpu
    blocks = 5000   # of 1 MB
    d = fnpu.make_desc(64, 64, 128, 128, 64, blocks)
    k, v = (torch.empty((blocks, 64, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for x in (k, v):
        x[4998], x[1], x[4100] = torch.randn_like(x[1]), torch.randn_like(x[1]), 0
    fnpu.kv_copy_blocks(d, _dev([[4998, 4100], [1, 4999]], np.int32), [k], [v])
    torch.cuda.synchronize()
    for x in (k, v):
        assert torch.equal(x[4100], x[4998]) and torch.equal(x[4999], x[1])
