"""Attention over the 8-bit block cache, held to a bound by each row's own weights.

The bound (``oracle.kv8.attention_bound``, where it is derived) is of the size of what
rounding the weights once does to that row, so that a block of values left out, or a scale
off by two, shows in every row that sees it (``test_oracle_kv8_bound`` plants both)."""
import numpy as np
import pytest

from oracle import kv8 as K8
from test_gpu_kv8 import FMTS, LAYOUTS, RAGGED, Cache, _bf16

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2606_04415_gb300 as fnpu
    fnpu.load()


def staged_sequences(c, ql, plan):
    """Sequences that a plan takes to the staged prefill: none where it has no prefill
    items, else those of more than 64 rows a kv head (middle chunks attend over the codes
    all together or not at all)."""
    return [plan.info()["prefill_items"] > 0 and n * (c.hq // c.hkv) > 64 for n in ql]


def check(c, ql, plan, q, out, lse, tokens=None):
    ref, ref_l, bound = K8.attention_bound(q.double().cpu().numpy(), ql, c.ctx, c.table, *c.pools, c.hkv, c.bs, c.d, c.fmt,
                                           staged_sequences(c, ql, plan), tokens=tokens)
    rows = np.arange(len(ref)) if tokens is None else np.array(sorted(tokens))
    o, l = out.double().cpu().numpy()[rows], lse.double().cpu().numpy()[rows]
    off = np.abs(o - ref[rows]) - bound[rows]
    assert (off <= 0).all(), (off.max(), rows[np.unravel_index(off.argmax(), off.shape)[0]])
    assert (np.abs(l - ref_l[rows]) <= 2e-5 * np.maximum(1, np.abs(ref_l[rows]))).all()


def run(c, ql, q=None, opts=None, plan=None, tokens=None):
    ql = np.asarray(ql, np.int32)
    T = int(ql.sum())
    q = _bf16(c.rng, T, c.hq, c.d).cuda() if q is None else q
    if plan is None:
        plan = c.fnpu.kv8_attn_plan(c.desc, c.fmt, ql, c.ctx, (ql == 1).astype(np.uint8), c.table, opts=opts)
    out = torch.full((T, c.hq, c.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, c.hq), float("nan"), device="cuda")
    c.fnpu.mixed_attn_run(plan, q, *c.dev, out, lse)
    assert c.fnpu.plan_check(plan) == c.fnpu.FNPU_OK and c.fnpu.check() == c.fnpu.FNPU_OK
    check(c, ql, plan, q, out, lse, tokens)
    return plan, q, out, lse


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs", LAYOUTS)
def test_decode(fmt, hq, hkv, d, bs):
    c = Cache(RAGGED, hq, hkv, d, bs, fmt, seed=3 * hq + bs)
    c.fill(c.ctx)
    run(c, np.ones(len(RAGGED)))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs", [(28, 4, 128, 16), (4, 2, 64, 32), (8, 1, 64, 64)])
@pytest.mark.parametrize("split", [16, 112, 0])
def test_several_tokens_in_pieces(fmt, hq, hkv, d, bs, split):
    """More than twelve pieces of a sequence too (their partial results are merged in groups)."""
    import paper_2606_04415_gb300 as fnpu
    c = Cache([1, 17, 333, 641, 1700], hq, hkv, d, bs, fmt, seed=split + 1)
    c.fill(c.ctx)
    run(c, [1, 2, 5, 8, 4], opts=fnpu.PlanOpts(split, 0, 0, 0))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,q", [(8, 1, 64, 250), (4, 2, 64, 700), (28, 4, 128, 60), (40, 1, 128, 33)])
def test_middle_chunks(fmt, hq, hkv, d, q):
    c = Cache([q + 50, q, q + 900], hq, hkv, d, 16, fmt, seed=q + 1)
    c.fill(c.ctx)
    rows = set(c.rng.permutation(3 * q)[:16].tolist()) | {0, q - 1, q, 2 * q - 1, 2 * q, 3 * q - 1}
    plan, *_ = run(c, [q, q, q], tokens=rows)
    assert plan.info()["prefill_items"] == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv,d,bs,n", [(28, 4, 128, 16, 400), (4, 2, 64, 32, 1500), (32, 8, 128, 64, 1300), (8, 1, 64, 16, 1025)])
def test_staged_chunks(fmt, hq, hkv, d, bs, n):
    """Beside a middle chunk, a short one and a decode; and on a long prefix."""
    ql = [n, 100, 2, 1]
    c = Cache([n + 77, 150, 40, 500], hq, hkv, d, bs, fmt, seed=n + 2)
    c.fill(c.ctx)
    plan, *_ = run(c, ql, tokens={0, 130, n - 1, n, n + 99, n + 100, n + 101, n + 102})
    info = plan.info()
    assert info["prefill_items"] > 0 and info["decode_items"] > 0
    one = Cache([n + 3000], hq, hkv, d, bs, fmt, seed=n + 3)
    one.fill(one.ctx)
    plan, *_ = run(one, [n], tokens={0, n // 2, n - 1})
    assert plan.info()["prefill_items"] > 0 and plan.info()["decode_items"] == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_long_context(fmt):
    c = Cache([40011, 3, 900], 7, 1, 128, 64, fmt, seed=24)
    c.fill(c.ctx)
    run(c, [2, 1, 1])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("ql", [1, 40])
def test_scales_far_apart(fmt, ql):
    """Values of blocks 2^40 apart in size. Half of the queries point at a key (their
    product with it is some 60 above the others'), mostly of small blocks: what decides
    the result there are values far below the largest of the cache."""
    c = Cache([2000, 333, 64], 8, 2, 128, 16, fmt, seed=22 + ql)
    n = int(c.ctx.sum())
    sl = np.concatenate([c.slots(s, 0, int(x)) for s, x in enumerate(c.ctx)])
    k, v = c.rows(n, 0.0), c.rows(n)
    size = c.rng.integers(-20, 21, (n // 16 + 1, 2, 1))
    v = (v.double() * torch.from_numpy(np.exp2(size).repeat(16, 0)[:n])).to(torch.bfloat16)
    c.append(k, v, sl)
    q = _bf16(c.rng, 3 * ql, 8, 128)
    first = np.concatenate([[0], np.cumsum(c.ctx)[:-1]])
    for s in range(3):
        for i in range(ql):
            for h in range(0, 8, 2):
                see = int(c.ctx[s]) - ql + i + 1
                j = first[s] + c.rng.integers(0, see, 8)
                j = j[size[j // 16, h // 4, 0].argmin()]
                q[s * ql + i, h] = k[j, h // 4] * 8
    tokens = None if ql == 1 else {0, 1, 20, 39, 40, 60, 79, 80, 99, 119}
    plan, *_ = run(c, [ql] * 3, q=q.cuda(), tokens=tokens)
    assert plan.info()["prefill_items"] == 0
