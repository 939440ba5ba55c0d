"""Forks of states whose counts are lower than their pages' holders: flagged where the
header says so, and the same result every time."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BS = 16


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype))).cuda()


def _fork(table, n, refs, parents, grow):
    """(what check gives, refs, new table, lengths, slots, copies, stats) as lists."""
    import paper_2606_04415_gb300 as fnpu
    table, refs = np.asarray(table, np.int32), _dev(refs)
    new = len(n) if parents is None else len(parents)
    d = fnpu.make_pages(BS, len(refs))
    out = [torch.full(s, 77, dtype=t, device="cuda") for s, t in (((new, table.shape[1]), torch.int32), ((new,), torch.int32),
                                                                  ((new, grow), torch.int64), ((new, 2), torch.int32), ((4,), torch.int32))]
    ws = torch.randint(0, 256, (fnpu.pages_workspace(d, new),), dtype=torch.uint8, device="cuda")
    fnpu.pages_fork(d, _dev(table), _dev(n), refs, *out, ws, parents=None if parents is None else _dev(parents))
    return fnpu.check(), refs.tolist(), *(x.tolist() for x in out)


@pytest.mark.parametrize("blocks,others", [(40, 0), (2048, 60), (9000, 100)])
@pytest.mark.parametrize("count", [1, 2, 3, 4])
def test_last_pages_with_fewer_holders_counted(blocks, others, count):
    """Three rows share a partly filled last page whose count is `count`: below three it is
    flagged and stays, and two rows copy all the same. One CTA, and several chunks of counts
    (the page in one whose free blocks another CTA hands out)."""
    import paper_2606_04415_gb300 as fnpu
    page, first = blocks - 3, 1
    table = np.full((3 + others, 3), -1, np.int32)
    table[:3, 0], table[:3, 1] = 0, page
    table[3:, 0] = np.arange(first, first + others)
    n = np.array([20] * 3 + [BS] * others, np.int32)         # (the others' pages are full: each takes a new one)
    refs = np.zeros(blocks, np.int32)
    refs[0], refs[page], refs[first:first + others] = 3, count, 1
    free = [b for b in range(blocks) if refs[b] == 0]
    copying = [0, 1, 2] if count == 4 else [1, 2]
    for _ in range(10):
        flag, got, rows, lens, slots, copies, stats = _fork(table, n, refs, None, 1)
        assert flag == (fnpu.FNPU_EDEVICE_RANGE if count < 3 else 0)
        assert lens == [21] * 3 + [BS + 1] * others and stats == [len(free) - len(copying) - others, len(copying) + others, 0, len(copying)]
        take = iter(free)
        want, pairs = table.copy(), [[-1, -1]] * (3 + others)
        for r in copying:
            want[r, 1] = next(take)
            pairs[r] = [page, want[r, 1]]
        for r in range(3, 3 + others):
            want[r, 1] = next(take)
        assert rows == want.tolist() and copies == pairs
        assert slots == [[int(want[r, 1]) * BS + int(n[r]) % BS] for r in range(3 + others)]
        after = refs.copy()
        after[want[copying + list(range(3, 3 + others)), 1]] = 1
        after[page] = count if count < 3 else count - len(copying)
        assert got == after.tolist()
    assert fnpu.check() == 0


def test_a_last_page_that_nobody_counts():
    import paper_2606_04415_gb300 as fnpu
    table, refs = [[5, 9]], np.zeros(12, np.int32)
    refs[5] = 1
    flag, got, rows, lens, slots, copies, stats = _fork(table, [20], refs, None, 1)
    assert flag == fnpu.FNPU_EDEVICE_RANGE and rows == table and slots == [[9 * BS + 4]] and copies == [[-1, -1]]
    assert got == refs.tolist() and lens == [21] and stats == [11, 0, 0, 0]


@pytest.mark.parametrize("blocks,width", [(300, 100), (9000, 500)])
@pytest.mark.parametrize("count", [0, 1, 2, 5])
def test_holders_come_and_go_in_one_sum(blocks, width, count):
    """Pages of two rows, one given up and the other continued by three, with too low counts
    among them: the new count is the old one and one, whichever row's comes first; where the
    sum is below zero it is flagged and the count is zero."""
    import paper_2606_04415_gb300 as fnpu
    pages = np.arange(1, width + 1)
    refs = np.zeros(blocks, np.int32)
    refs[pages] = count
    for _ in range(10):
        for rows in (2, 40):                                   # (the first two rows' pages; those of the others are their own)
            table = np.full((rows, width), -1, np.int32)
            table[:2] = pages
            n = np.array([width * BS] * 2 + [0] * (rows - 2), np.int32)
            flag, got, new, lens, _, _, stats = _fork(table, n, refs, [1, 1, 1], 0)
            assert flag == 0 and np.array_equal(got, np.where(refs + np.isin(np.arange(blocks), pages) > 0, count + 1, 0))
            assert new == [pages.tolist()] * 3 and lens == [width * BS] * 3
            live = width if count + 1 > 0 else 0
            assert stats == [blocks - live, 0, 0, 0]
            flag, got, new, *_ = _fork(table, n, refs, [-1], 0)
            assert flag == (fnpu.FNPU_EDEVICE_RANGE if count < 2 else 0)
            assert np.array_equal(got, np.maximum(refs - 2 * np.isin(np.arange(blocks), pages), 0)) and new == [[-1] * width]
    assert fnpu.check() == 0
