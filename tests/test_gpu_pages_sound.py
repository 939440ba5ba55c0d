"""Forks of sound states raise no flag, whatever stands past their rows' pages."""
import os
import importlib.util

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("pages_states", os.path.join(os.path.dirname(os.path.abspath(__file__)), "test_gpu_pages.py"))
pages = importlib.util.module_from_spec(spec)
spec.loader.exec_module(pages)


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("rows,new,width,bs,blocks,grow", [(4, 4, 9, 16, 60, 1), (1, 8, 3, 4, 5, 2), (9, 3, 20, 1, 200, 5), (8, 8, 130, 64, 1100, 1),
                                                           (3, 12, 7, 32, 40, 100), (600, 700, 5, 16, 20000, 1), (5, 5, 6, 16, 40, 0),
                                                           (2, 5000, 4, 16, 9000, 1)])
def test_fork(seed, rows, new, width, bs, blocks, grow):
    st = pages.State(seed, rows, width, bs, blocks, most=max(1, width * bs - (grow if seed % 2 else 0)), freed=0.1 * (seed % 2))
    parents = st.rng.integers(-1 if seed % 3 else 0, rows, new)
    refs, got = pages._dev(st.refs, np.int32), pages._outputs(st, new, grow)
    st.fnpu.pages_fork(st.desc, st.table(), pages._dev(st.n, np.int32), refs, *got, st.workspace(max(rows, new)), parents=pages._dev(parents, np.int32))
    assert st.fnpu.check() == 0
    pages._check_fork(st, parents.tolist(), grow, got, refs)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows,blocks", [(30, 400), (200, 6000)])
def test_fork_of_the_same_rows(rows, blocks, in_place):
    st = pages.State(5, rows, 10, 16, blocks, most=150)
    refs, got, table, n = pages._dev(st.refs, np.int32), list(pages._outputs(st, rows, 3)), st.table(), pages._dev(st.n, np.int32)
    if in_place:
        got[0], got[1] = table, n
    st.fnpu.pages_fork(st.desc, table, n, refs, *got, st.workspace(rows))
    assert st.fnpu.check() == 0
    pages._check_fork(st, list(range(rows)), 3, got, refs)
