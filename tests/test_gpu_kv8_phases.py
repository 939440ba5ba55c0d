"""Steps over the 8-bit block cache whose chunks are staged for the tensor-core prefill:
the ways of running both phases, the options that ask for one, and re-plans between a
staged step and others.

Tolerances as in ``test_gpu_kv8_bound``; a chunk of more than 2048 rows a kv head (query tokens
times query heads of it) is staged whatever the planner's model says."""
import numpy as np
import pytest

from oracle import kv8 as K8
from test_gpu_kv8 import FMTS, Cache, _bf16, _compare
from test_gpu_kv8_bound import check, run

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


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs,chunk", [(28, 4, 128, 16, 310), (4, 2, 64, 32, 1100), (32, 8, 128, 64, 530), (8, 1, 64, 16, 270)])
def test_both_phases_in_every_way(fmt, hq, hkv, d, bs, chunk):
    """A staged chunk, a middle one, a short one and decodes: as planned, with separate
    launches, with a share asked for and in green contexts; run twice each."""
    import paper_2606_04415_gb300 as fnpu
    ql, ctx = [chunk, 90, 2, 1, 1, 1], [chunk + 100, 95, 33, 700, 18, 1]
    c = Cache(ctx, hq, hkv, d, bs, fmt, seed=chunk)
    c.fill(c.ctx)
    q = _bf16(c.rng, sum(ql), hq, d).cuda()
    rows = set(c.rng.permutation(chunk)[:6].tolist()) | {0, chunk - 1, chunk, chunk + 89, chunk + 90, chunk + 91} | set(range(chunk + 92, chunk + 95))
    for flags, pct, together in ((0, 0, None), (fnpu.PLAN_SEPARATE_LAUNCHES, 0, False), (0, 10, True), (fnpu.PLAN_GREEN_CONTEXTS, 0, True),
                                 (fnpu.PLAN_GREEN_CONTEXTS, 20, True)):
        try:
            plan = _plan(c, ql, fnpu.PlanOpts(0, pct, 0, flags))
        except fnpu.FnpuError as e:
            assert flags == fnpu.PLAN_GREEN_CONTEXTS and e.code == fnpu.FNPU_EUNSUPPORTED
            continue
        info = plan.info()
        assert info["prefill_items"] > 0 and info["decode_items"] > 0
        if together is False:
            with pytest.raises(fnpu.FnpuError):
                fnpu.plan_decode_share(plan)
        elif together or hkv == 4:  # (four kv heads co-locate always)
            assert fnpu.plan_decode_share(plan) == (pct if pct and not flags else pytest.approx(25, abs=25))
        out, lse = _run(c, plan, q)
        check(c, ql, plan, q, out, lse, rows)
        again, lse2 = _run(c, plan, q)
        assert torch.equal(again, out) and torch.equal(lse2, lse)
        if together:
            assert min(fnpu.plan_phase_ms(plan)) > 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("prefix", [0, 500])
def test_rows_either_side_of_the_limit(fmt, prefix):
    """2048 rows a kv head may attend over the codes; 2056 never do."""
    for n, direct in ((256, True), (257, False)):
        c = Cache([n + prefix], 8, 1, 64, 16, fmt, seed=n)
        c.fill(c.ctx)
        plan, *_ = run(c, [n], tokens={0, 1, n // 2, n - 2, n - 1})
        assert (plan.info()["prefill_items"] == 0) == direct


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("flags", [0, 1])
def test_replan_between_staged_steps_and_others(fmt, flags):
    """One plan through a staged chunk, decodes alone, a middle chunk, a larger staged chunk
    (its workspace grows) and a small one again."""
    import paper_2606_04415_gb300 as fnpu
    plan = None
    for i, (ql, ctx) in enumerate((([300, 1], [340, 77]), ([1, 1, 1], [341, 78, 500]), ([100, 1], [130, 79]),
                                   ([900, 300, 1, 1], [1700, 301, 80, 12]), ([270, 2], [270, 9]))):
        c = Cache(ctx, 8, 1, 64, 16, fmt, seed=50 + i, blocks=200)
        c.fill(c.ctx)
        meta = (np.array(ql, np.int32), c.ctx, (np.array(ql) == 1).astype(np.uint8), c.table)
        opts = fnpu.PlanOpts(0, 0, 0, flags)
        if plan is None:
            plan = fnpu.kv8_attn_plan(c.desc, fmt, *meta, opts=opts)
        else:
            fnpu.mixed_attn_replan(plan, *meta, opts=opts)
        assert (plan.info()["prefill_items"] > 0) == (i in (0, 3, 4))
        T = sum(ql)
        run(c, ql, plan=plan, tokens=set(range(0, T, 97)) | {ql[0] - 1, ql[0], T - 1})


def test_staged_blocks_past_4_gb():
    """A staged chunk whose blocks lie on both sides of 2^32 bytes of the pools."""
    import paper_2606_04415_gb300 as fnpu
    hq, hkv, d, bs, fmt, ql = 16, 8, 128, 64, K8.INT8, 1030
    b = K8.block_bytes(hkv, bs, d)
    blocks = (1 << 32) // b + 40
    if torch.cuda.mem_get_info()[0] < 3 * blocks * b:
        pytest.skip("needs 13 GB of device memory")
    rng = np.random.default_rng(42)
    nb, ctx = 21, 21 * bs - 9
    ids = np.where(np.arange(nb) % 2, blocks - 1 - np.arange(nb), np.arange(nb) + 3).astype(np.int32)[None]
    pos = np.arange(ctx)
    sl = ids[0, pos // bs].astype(np.int64) * bs + pos % bs
    desc = fnpu.make_desc(hq, hkv, d, d, bs, blocks)
    dev = [torch.zeros(blocks * b, dtype=torch.uint8, device="cuda") for _ in range(2)]
    k, v = (_bf16(rng, ctx, hkv, d) for _ in range(2))
    fnpu.rope_append(desc, None, None, None, None, k.cuda(), v.cuda(), torch.from_numpy(sl).cuda(), None, *dev, kv_format=fmt)
    pools = [np.zeros(nb * b, np.uint8) for _ in range(2)]
    for pool, x in zip(pools, (k, v)):
        K8.append(pool, x.double().numpy(), np.arange(ctx), hkv, bs, d, fmt)
    q = _bf16(rng, ql, hq, d).cuda()
    out, lse = torch.empty((ql, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((ql, hq), device="cuda")
    plan = fnpu.kv8_attn_plan(desc, fmt, [ql], [ctx], [0], ids)
    assert plan.info()["prefill_items"] > 0 and plan.info()["decode_items"] == 0
    fnpu.mixed_attn_run(plan, q, *dev, out, lse)
    assert fnpu.plan_check(plan) == fnpu.FNPU_OK and fnpu.check() == fnpu.FNPU_OK
    rows = np.array([0, 1, 400, ql - 2, ql - 1])
    ref, ref_l, bound = K8.attention_bound(q.double().cpu().numpy(), [ql], [ctx], np.arange(nb)[None], *pools, hkv, bs, d, fmt, [True],
                                           tokens=set(rows.tolist()))
    assert (np.abs(out.double().cpu().numpy() - ref)[rows] <= bound[rows]).all()
    assert (np.abs(lse.double().cpu().numpy() - ref_l)[rows] <= 2e-5 * np.maximum(1, np.abs(ref_l[rows]))).all()
