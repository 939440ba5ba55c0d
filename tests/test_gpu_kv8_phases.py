"""Steps over the 8-bit block cache whose chunks are staged for the tensor-core prefill:
the ways of running both phases, the options that ask for one, and re-plans between a
staged step and others.

Tolerances as in ``test_gpu_kv8``; a chunk of more than 2048 rows a kv head (query tokens
times query heads of it) is staged whatever the planner's model says."""
import numpy as np
import pytest

from oracle import kv8 as K8
from test_gpu_kv8 import FMTS, Cache, _attend, _bf16, _compare

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def _plan(c, ql, opts=None):
    ql = np.array(ql, np.int32)
    return c.fnpu.kv8_attn_plan(c.desc, c.fmt, ql, c.ctx, (ql == 1).astype(np.uint8), c.table, opts=opts)


def _run(c, plan, q):
    T = q.shape[0]
    out = torch.full((T, c.hq, c.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, c.hq), float("nan"), device="cuda")
    c.fnpu.mixed_attn_run(plan, q, *c.dev, out, lse)
    assert c.fnpu.plan_check(plan) == c.fnpu.FNPU_OK and c.fnpu.check() == c.fnpu.FNPU_OK
    return out, lse


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs,chunk", [(28, 4, 128, 16, 60), (4, 2, 64, 32, 300), (32, 8, 128, 64, 200)])
def test_options_reach_middle_chunks(fmt, hq, hkv, d, bs, chunk):
    """A share of the SMs or green contexts asked for: chunks that would attend over the
    codes beside the decodes keep their own phase, and its share and times can be read."""
    import paper_2606_04415_gb300 as fnpu
    ql, ctx = [chunk, 1, 1, 3], [chunk + 100, 300, 77, 200]
    c = Cache(ctx, hq, hkv, d, bs, fmt, seed=chunk)
    c.fill(c.ctx)
    q = _bf16(c.rng, sum(ql), hq, d).cuda()
    for opts, share in ((fnpu.PlanOpts(0, 20, 0, 0), 20), (fnpu.PlanOpts(0, 0, 0, fnpu.PLAN_GREEN_CONTEXTS), None),
                        (fnpu.PlanOpts(0, 30, 0, fnpu.PLAN_GREEN_CONTEXTS), None)):
        try:
            plan = _plan(c, ql, opts)
        except fnpu.FnpuError as e:
            assert opts.flags == fnpu.PLAN_GREEN_CONTEXTS and e.code == fnpu.FNPU_EUNSUPPORTED
            continue
        assert plan.info()["prefill_items"] > 0 and plan.info()["decode_items"] > 0
        got = fnpu.plan_decode_share(plan)
        assert got == share if share else got > 0
        out, lse = _run(c, plan, q)
        _compare(c, ql, q, out, lse)
        assert min(fnpu.plan_phase_ms(plan)) > 0
    plan = _plan(c, ql)  # without: over the codes
    assert plan.info()["prefill_items"] == 0
    out, lse = _run(c, plan, q)
    _compare(c, ql, q, out, lse)
