"""Refusals of the rotary and 8-bit cache entry points, decided on the host (no
GPU), and their plans' checks."""
import ctypes

import numpy as np
import pytest

import paper_2606_04415_gb300 as fnpu

SHAPE = dict(num_q_heads=28, num_kv_heads=4, head_dim_qk=128, head_dim_v=128, block_size=16, num_blocks=100)
INV, UNS, OK = fnpu.FNPU_EINVAL, fnpu.FNPU_EUNSUPPORTED, fnpu.FNPU_OK


def _rope(rope=None, inv=64, pos=128, x=256, xs=3584, heads=28, d=128, n=5, out=4096, os=3584):
    rope = fnpu.make_rope(128) if rope is None else rope
    return fnpu.load().fnpu_rope(ctypes.byref(rope), inv, pos, x, xs, heads, d, n, out, os, None)


@pytest.mark.parametrize("kw", [dict(inv=None), dict(inv=68), dict(pos=None), dict(pos=130), dict(x=None), dict(x=257),
                                dict(out=None), dict(xs=3583), dict(os=100), dict(heads=0), dict(d=64), dict(n=-1), dict(x=4096, xs=4000)])
def test_rope_rejects(kw):
    assert _rope(**kw) == INV


def test_rope_descriptor():
    assert _rope(n=0) == OK
    for bad in (dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=-2), dict(rotary_dim=130), dict(rotary_dim=64, rotary_offset=65),
                dict(rotary_dim=64, rotary_offset=-1), dict(rotary_dim=64, rotary_offset=2**31 - 1), dict(rotary_dim=64, num_axes=0),
                dict(rotary_dim=64, num_axes=5, pair_axis=np.zeros(32)), dict(rotary_dim=64, num_axes=2),
                dict(rotary_dim=64, num_axes=2, pair_axis=np.full(32, 2))):
        assert _rope(fnpu.make_rope(**bad)) == INV, bad
    r = fnpu.make_rope(64)
    r.interleaved = 2
    assert _rope(r) == INV
    r.interleaved, r.inverse = 0, -1
    assert _rope(r) == INV
    assert fnpu.load().fnpu_rope(None, 64, 128, 256, 3584, 28, 128, 5, 4096, 3584, None) == INV
    assert _rope(fnpu.make_rope(258), heads=1, d=512, xs=512, os=512) == UNS
    with pytest.raises(ValueError):
        fnpu.make_rope(64, num_axes=2, pair_axis=np.zeros(31))


def _append(desc=None, fmt=fnpu.KV_INT8_BLOCK, rope=True, q=256, qs=3584, k=512, ks=512, v=1024, vs=512, slots=2048, n=4, qo=4096,
            kc=8192, vc=16384, **r):
    desc = fnpu.make_desc(**SHAPE) if desc is None else desc
    rd = fnpu.make_rope(**dict(dict(rotary_dim=128), **r)) if rope else None
    return fnpu.load().fnpu_rope_append(ctypes.byref(desc), fmt, None if rd is None else ctypes.byref(rd), 64, 128, q, qs, k, ks, v, vs,
                                        slots, n, qo, kc, vc, None)


@pytest.mark.parametrize("fmt", [fnpu.KV_BF16, fnpu.KV_INT8_BLOCK, fnpu.KV_E4M3_BLOCK])
@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(slots=None), dict(kc=None), dict(vc=None), dict(k=520), dict(v=1032),
                                dict(q=264), dict(qo=None), dict(qo=4104), dict(slots=2052), dict(kc=8200), dict(ks=511), dict(ks=516),
                                dict(vs=100), dict(qs=3583), dict(qs=3588), dict(n=-1), dict(rope=False), dict(q=4096, qs=4096)])
def test_append_rejects(fmt, kw):
    assert _append(fmt=fmt, **kw) == INV


def test_append_formats_and_shapes():
    assert _append(n=0) == OK and _append(n=0, fmt=fnpu.KV_BF16) == OK
    assert _append(fmt=3) == INV and _append(fmt=-1) == INV
    bad = fnpu.make_desc(**SHAPE)
    bad.kv_fp8 = 2
    assert _append(bad) == INV
    for other in (dict(head_dim_v=64), dict(head_dim_qk=64), dict(block_size=8), dict(block_size=128), dict(block_size=48),
                  dict(head_dim_qk=192, head_dim_v=192)):
        assert _append(fnpu.make_desc(**dict(SHAPE, **other)), ks=1 << 20, vs=1 << 20, qs=1 << 20) == UNS, other
    for fmt in (0, 1, 2):
        assert _append(fnpu.make_desc(**SHAPE, kv_fp8=True), fmt=fmt) == UNS
    assert _append(fnpu.make_desc(128, 1, 576, 512, 64, 8, latent=True)) == UNS
    assert _append(rotary_dim=24) == UNS
    assert _append(rotary_dim=64, rotary_offset=8) == UNS          # 8-bit rows turn in groups of 16 columns
    assert _append(rotary_dim=64, rotary_offset=4, fmt=0) == UNS
    assert _append(rope=False, q=None, fmt=0, ks=520) == UNS       # strided rows without a rotation


def test_read_rejects():
    lib = fnpu.load()
    desc = fnpu.make_desc(**SHAPE)
    ok = [16, 4, 64, 128, 256, 512]

    def call(fmt=1, d=desc, **kw):
        a = list(ok)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return lib.fnpu_kv_read(ctypes.byref(d), fmt, *a, None)
    for fmt in (0, 1, 2):
        assert call(fmt, a1=0) == OK
        for bad in (dict(a0=None), dict(a0=12), dict(a1=-1), dict(a2=None), dict(a2=72), dict(a3=None), dict(a4=None), dict(a4=264),
                    dict(a5=None), dict(a5=520)):
            assert call(fmt, **bad) == INV, (fmt, bad)
    assert call(3) == INV and call(1, fnpu.make_desc(**SHAPE, kv_fp8=True)) == UNS


def test_block_bytes():
    assert fnpu.kv8_block_bytes(fnpu.make_desc(**SHAPE), fnpu.KV_INT8_BLOCK) == 16 * 4 * 128 + 16
    assert fnpu.kv8_block_bytes(fnpu.make_desc(12, 6, 64, 64, 64, 3), fnpu.KV_E4M3_BLOCK) == 64 * 6 * 64 + 32
    for desc, fmt, code in ((fnpu.make_desc(**SHAPE), fnpu.KV_BF16, INV), (fnpu.make_desc(**dict(SHAPE, block_size=8)), 1, UNS)):
        with pytest.raises(fnpu.FnpuError) as e:
            fnpu.kv8_block_bytes(desc, fmt)
        assert e.value.code == code
    assert fnpu.load().fnpu_kv8_block_bytes(ctypes.byref(fnpu.make_desc(**SHAPE)), 1, None) == INV


def _plan_rc(desc, fmt=1, ql=(4, 1), cl=(10, 40), ph=(0, 1), bt=None, opts=None):
    bt = np.zeros((2, 4), np.int32) if bt is None else bt
    arrays = [np.asarray(a, t) for a, t in ((ql, np.int32), (cl, np.int32), (ph, np.uint8))]
    out = ctypes.c_void_p()
    return fnpu.load().fnpu_kv8_attn_plan(ctypes.byref(desc), fmt, len(ql), *(a.ctypes.data for a in arrays), bt.ctypes.data, bt.shape[1],
                                          None if opts is None else ctypes.byref(opts), None, ctypes.byref(out))


def test_plan_rejects():
    d = fnpu.make_desc(**SHAPE)
    assert _plan_rc(d, fmt=0) == INV and _plan_rc(d, fmt=3) == INV
    assert _plan_rc(d, cl=(3, 40)) == INV and _plan_rc(d, ql=(0, 1)) == INV and _plan_rc(d, ph=(0, 2)) == INV
    bt = np.zeros((2, 4), np.int32)
    bt[1, 2] = 100
    assert _plan_rc(d, bt=bt) == INV
    assert _plan_rc(d, bt=np.zeros((2, 2), np.int32)) == INV
    for other in (dict(block_size=8), dict(head_dim_v=64), dict(num_q_heads=4 * 129), dict(block_size=128)):
        assert _plan_rc(fnpu.make_desc(**dict(SHAPE, **other)), bt=np.zeros((2, 8), np.int32)) == UNS, other
    assert _plan_rc(fnpu.make_desc(**SHAPE, kv_fp8=True)) == UNS
    assert _plan_rc(fnpu.make_desc(128, 1, 576, 512, 64, 100, latent=True), ph=(0, 1)) == UNS
    assert _plan_rc(d, opts=fnpu.PlanOpts(0, 0, 0, fnpu.PLAN_NO_TCGEN05)) == UNS
    # valid shapes (without a GPU they fail later)
    for hq, hkv, dim in ((4, 2, 64), (8, 1, 64), (32, 8, 128), (6, 3, 128), (40, 1, 128), (16, 16, 128)):
        assert _plan_rc(fnpu.make_desc(hq, hkv, dim, dim, 32, 100)) not in (INV, UNS)
