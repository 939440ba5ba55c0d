"""A windowed step run in every way: together, in launches of its own, in green contexts."""
import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("window_steps", os.path.join(os.path.dirname(os.path.abspath(__file__)), "test_gpu_window.py"))
steps = importlib.util.module_from_spec(spec)
spec.loader.exec_module(steps)


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


@pytest.mark.parametrize("window,sinks", [(60, 4), (700, 0), (128, 300)])
def test_runs_repeat_and_ways_agree(window, sinks):
    """Each way gives the same bits every time. Ways differ by where pieces are cut alone, so
    their rows lie within the sum of both bounds of each other."""
    from oracle import window as W
    st = steps.Step((28, 4, 128), 16, [(200, 900, 0), (1, 700, 1), (1, 1, 1), (90, 90, 0), (1, 333, 1), (4, 600, 1)], window, sinks, seed=11)
    outs = []
    for flags in (0, st.fnpu.PLAN_SEPARATE_LAUNCHES, st.fnpu.PLAN_GREEN_CONTEXTS):
        plan = st.plan(st.fnpu.PlanOpts(0, 0, 0, flags))
        runs = []
        for _ in range(3):
            st.out.fill_(7.0), st.lse.fill_(7.0)
            st.run(plan)
            runs.append((st.out.clone(), st.lse.clone()))
        st.check()
        assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))
        outs.append([x.float().cpu().numpy() for x in runs[0]])
    q, k, v = (x.float().cpu().numpy() for x in (st.q, st.k, st.v))
    at = 0
    for s, (n, c) in enumerate(zip(st.q_len, st.ctx)):
        ref = W.attend(q[at:at + n], k, v, st.table[s], int(c - n), st.bs, window, sinks)
        bounds = W.bounds(*ref, q.shape[2])
        for other in outs[1:]:
            for x, y, b in zip(outs[0], other, bounds):
                assert (np.abs(x[at:at + n] - y[at:at + n]) <= 2 * b).all(), f"sequence {s}"
        at += n
