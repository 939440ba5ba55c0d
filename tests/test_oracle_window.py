"""Pins of the windowed attention reference, and what plans and calls refuse."""
import ctypes

import numpy as np
import pytest

import oracle
import paper_2606_04415_gb300 as fnpu
from oracle import window as W


def _case(seed, ctx, hq=4, hkv=2, d=8, bs=4):
    rng = np.random.default_rng(seed)
    nb = -(-ctx // bs)
    table = rng.permutation(nb + 3)[:nb]
    return rng.standard_normal((ctx, hq, d)), rng.standard_normal((nb + 3, bs, hkv, d)), rng.standard_normal((nb + 3, bs, hkv, d)), table


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (3, 0), (3, 2), (7, 5), (40, 0), (4, 60)])
def test_visible_keys_by_counting(window, sinks):
    for p in range(30):
        seen = W.visible(p, window, sinks)
        lo = max(0, p - window + 1)
        assert seen == sorted(set(range(min(sinks, p + 1))) | set(range(lo, p + 1)))


def test_one_key_gives_its_value():
    q, k, v, t = _case(1, 9)
    out, lse, _, _ = W.attend(q[8:], k, v, t, 8, 4, 1, 0)
    for h in range(4):
        assert np.allclose(out[0, h], v[t[2], 0, h // 2])
        assert np.allclose(lse[0, h], q[8, h] @ k[t[2], 0, h // 2] / 8 ** 0.5)


def test_wide_window_is_causal_attention():
    """Against the C reference of the causal step."""
    rng = np.random.default_rng(2)
    bits = [(rng.standard_normal(s).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
            for s in ((11, 4, 64), (6, 16, 2, 64), (6, 16, 2, 64))]
    t = np.array([[4, 0, 5, 2]], np.int32)
    o, l = oracle.attention(np.array([11], np.int32), np.array([50], np.int32), t, *bits, num_q_heads=4, num_kv_heads=2, head_dim_qk=64, head_dim_v=64,
                            block_size=16)
    f = [(x.astype(np.uint32) << 16).view(np.float32) for x in bits]
    for window, sinks in ((50, 0), (1, 50), (20, 40)):
        out, lse, _, _ = W.attend(*f, t[0], 39, 16, window, sinks)
        assert np.allclose(out, o, atol=1e-12) and np.allclose(lse, l, atol=1e-12)


def test_window_equals_attention_over_the_cut_sequence():
    """Without sinks, the window of a query is a sequence of its own."""
    q, k, v, t = _case(3, 33)
    out, lse, _, _ = W.attend(q[32:], k, v, t, 32, 4, 13, 0)
    flat = k[t].reshape(-1, 2, 8)[20:33], v[t].reshape(-1, 2, 8)[20:33]
    one = [np.concatenate([x, np.zeros((3, 2, 8))]).reshape(4, 4, 2, 8) for x in flat]
    o2, l2, _, _ = W.attend(q[32:], *one, np.arange(4), 12, 4, 1000, 0)
    assert np.allclose(out, o2, atol=1e-13) and np.allclose(lse, l2, atol=1e-13)


def test_sinks_and_window_merge_by_log_sum_exp():
    q, k, v, t = _case(4, 33)
    both = W.attend(q[32:], k, v, t, 32, 4, 10, 5)
    near = W.attend(q[32:], k, v, t, 32, 4, 10, 0)
    sink = W.attend(q[32:], k, v, t, 4, 4, 5, 0)   # keys 0 .. 4
    total = np.logaddexp(near[1], sink[1])
    assert np.allclose(both[1], total, atol=1e-13)
    mix = near[0] * np.exp(near[1] - total)[..., None] + sink[0] * np.exp(sink[1] - total)[..., None]
    assert np.allclose(both[0], mix, atol=1e-13)


def test_hidden_rows_do_not_matter():
    q, k, v, t = _case(5, 33)
    ref = W.attend(q[30:], k, v, t, 30, 4, 6, 3)
    for j in range(3, 25):
        k[t[j // 4], j % 4], v[t[j // 4], j % 4] = np.nan, np.inf
    t = np.array(t)
    t[1:6] = -1
    for a, b in zip(ref, W.attend(q[30:], k, v, t, 30, 4, 6, 3)):
        assert np.array_equal(a, b)


# --------------------------------------------------------------- refusals

def _rc(desc, window, sinks, ql, cl, ph, bt, opts=None):
    ql, cl, ph, bt = (np.ascontiguousarray(a, t) for a, t in ((ql, np.int32), (cl, np.int32), (ph, np.uint8), (bt, np.int32)))
    out = ctypes.c_void_p()
    return fnpu.load().fnpu_window_attn_plan(ctypes.byref(desc), window, sinks, len(ql), ql.ctypes.data, cl.ctypes.data, ph.ctypes.data,
                                             bt.ctypes.data, bt.shape[1], None if opts is None else ctypes.byref(opts), None,
                                             ctypes.byref(out))


GOOD = dict(num_q_heads=4, num_kv_heads=2, head_dim_qk=64, head_dim_v=64, block_size=16, num_blocks=8)


def _desc(**kw):
    return fnpu.make_desc(**{**GOOD, **kw})


@pytest.mark.parametrize("window,sinks", [(0, 0), (-1, 4), (5, -1)])
def test_plan_refuses_windows(window, sinks):
    assert _rc(_desc(), window, sinks, [1], [40], [1], [[0, 1, 2]]) == fnpu.FNPU_EINVAL


@pytest.mark.parametrize("kw,phase", [(dict(kv_fp8=True, num_q_heads=28, num_kv_heads=4, head_dim_qk=128, head_dim_v=128), 1),
                                      (dict(latent=True, num_q_heads=64, num_kv_heads=1, head_dim_qk=576, head_dim_v=512), 1),
                                      (dict(head_dim_qk=192, head_dim_v=128), 0), (dict(block_size=24), 1), (dict(block_size=48), 0),
                                      (dict(num_q_heads=18), 1), (dict(head_dim_qk=96, head_dim_v=96), 0)])
def test_plan_refuses_caches(kw, phase):
    assert _rc(_desc(**kw), 10, 2, [1], [40], [phase], [[0, 1, 2]]) == fnpu.FNPU_EUNSUPPORTED


def test_plan_refuses_the_path_without_tcgen05():
    assert _rc(_desc(), 10, 2, [4], [40], [0], [[0, 1, 2]], fnpu.PlanOpts(0, 0, 0, fnpu.PLAN_NO_TCGEN05)) == fnpu.FNPU_EUNSUPPORTED


@pytest.mark.parametrize("entry,needed", [(0, True), (1, False), (2, False), (3, True), (4, True)])
def test_plan_checks_the_blocks_that_a_query_sees(entry, needed):
    """Contexts of 70: sinks in block 0, queries 68 and 69 with windows from 49 (block 3) on."""
    bt = np.array([[0, 1, 2, 3, 4]], np.int32)
    bt[0, entry] = -1
    rc = _rc(_desc(), 20, 3, [2], [70], [0], bt, fnpu.PlanOpts(0, 0, 1, 0))
    assert (rc == fnpu.FNPU_EINVAL) == needed
    bt[0, entry] = 8
    assert (_rc(_desc(), 20, 3, [2], [70], [0], bt, fnpu.PlanOpts(0, 0, 1, 0)) == fnpu.FNPU_EINVAL) == needed


def _decode_rc(desc, window=10, sinks=2, n=2, stride=3, most=40, split=0, q=1 << 20, ws=1 << 20, size=1 << 30):
    p = 1 << 20
    return fnpu.load().fnpu_window_decode(ctypes.byref(desc), window, sinks, n, p, p, stride, most, split, q, p, p, p, p, ws, size, None)


@pytest.mark.parametrize("kw", [dict(window=0), dict(sinks=-1), dict(n=-1), dict(stride=2), dict(most=-1), dict(split=32), dict(split=-64),
                                dict(q=None), dict(q=(1 << 20) + 8), dict(ws=(1 << 20) + 4)])
def test_decode_refuses_arguments(kw):
    assert _decode_rc(_desc(), **kw) == fnpu.FNPU_EINVAL


def test_decode_refuses_caches_and_small_workspaces():
    for kw in (dict(kv_fp8=True), dict(block_size=24), dict(num_q_heads=18), dict(head_dim_qk=96, head_dim_v=96), dict(head_dim_v=128)):
        assert _decode_rc(_desc(**kw)) == fnpu.FNPU_EUNSUPPORTED
    d = _desc()
    need = fnpu.window_decode_workspace(d, 1000, 4, 3, 5000, 128)
    assert need > 0
    assert _decode_rc(d, 1000, 4, 3, 400, 5000, 128, size=need - 1) == fnpu.FNPU_EINVAL
    assert _decode_rc(d, 1000, 4, 3, 400, 5000, 128, ws=None) == fnpu.FNPU_EINVAL
    # 16 keys of whole sink stages, the window and at most 15 ahead of it in its first stage: 131, 121
    assert fnpu.window_decode_workspace(d, 100, 4, 3, 5000, 128) > 0
    assert fnpu.window_decode_workspace(d, 90, 4, 3, 5000, 128) == 0     # one split: none needed
    assert fnpu.window_decode_workspace(d, 2 ** 31 - 1, 2 ** 31 - 1, 3, 5000, 512) == fnpu.window_decode_workspace(d, 5000, 0, 3, 5000, 512)
    with pytest.raises(fnpu.FnpuError):
        fnpu.window_decode_workspace(d, 0, 4, 3, 5000)
