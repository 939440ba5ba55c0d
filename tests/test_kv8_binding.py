"""What the binding of the rotary and 8-bit cache calls refuses or marshals before it
reaches the library (a stub stands in for it: no GPU, nothing is launched)."""
import numpy as np
import pytest

import paper_2606_04415_gb300 as fnpu

torch = pytest.importorskip("torch")

BF16, U8 = torch.bfloat16, torch.uint8
HQ, HKV, D, BS, BLOCKS, N = 4, 2, 64, 16, 5, 3
BLOCK = HKV * BS * D + 16


class Device:
    """A tensor's face without memory behind it."""
    is_cuda = True

    def __init__(self, *shape, dtype=BF16, stride=None, ptr=4096, contiguous=True):
        self.shape, self.dtype, self.ptr, self.contiguous = torch.Size(shape), dtype, ptr, contiguous
        self.strides = stride or torch.empty(shape, device="meta").stride()

    def numel(self):
        return self.shape.numel()

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return self.ptr


class Library:
    """Records calls; every one succeeds."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    stub = Library()
    monkeypatch.setattr(fnpu, "_lib", stub)
    return stub


def _desc(**kw):
    return fnpu.make_desc(**dict(dict(num_q_heads=HQ, num_kv_heads=HKV, head_dim_qk=D, head_dim_v=D, block_size=BS, num_blocks=BLOCKS), **kw))


def _bf16_pool(blocks=BLOCKS, **kw):
    return Device(blocks, BS, HKV, D, **kw)


def _byte_pool(size=BLOCKS * BLOCK, **kw):
    return Device(size, dtype=U8, **kw)


def _append(k_cache, v_cache, desc=None, **kw):
    rows = [Device(N, h, D) for h in (HQ, HKV, HKV)]
    fnpu.rope_append(desc or _desc(), fnpu.make_rope(D), Device(D // 2, dtype=torch.float32), Device(1, N, dtype=torch.int32), *rows,
                     Device(N, dtype=torch.int64), Device(N, HQ, D), k_cache, v_cache, stream=0, **kw)


def _read(k_cache, v_cache, desc=None, **kw):
    fnpu.kv_read(desc or _desc(), Device(N, dtype=torch.int64), k_cache, v_cache, Device(N, HKV, D), Device(N, HKV, D), stream=0, **kw)


GOOD = [(fnpu.KV_BF16, _bf16_pool), (fnpu.KV_INT8_BLOCK, _byte_pool), (fnpu.KV_E4M3_BLOCK, _byte_pool)]
BAD = [(fnpu.KV_BF16, _byte_pool()),                                  # the format left out over an 8-bit pool
       (fnpu.KV_BF16, _byte_pool(BLOCKS * BS * HKV * D * 2)),         # ... whatever its size
       (fnpu.KV_BF16, _bf16_pool(BLOCKS - 1)), (fnpu.KV_BF16, _bf16_pool(dtype=torch.float32)),
       (fnpu.KV_INT8_BLOCK, _bf16_pool()), (fnpu.KV_E4M3_BLOCK, _byte_pool(BLOCKS * BLOCK - 1)),
       (fnpu.KV_INT8_BLOCK, _byte_pool(BLOCKS * HKV * BS * D))]       # codes without their scales


@pytest.mark.parametrize("call", [_append, _read])
def test_pools_fit_their_format(lib, call):
    for fmt, pool in GOOD:
        call(pool(), pool(), kv_format=fmt)
        call(4096, 8192, kv_format=fmt)                               # raw addresses: the caller's
    assert len(lib.calls) == 6
    good = dict(GOOD)
    for fmt, bad in BAD:
        for pools in ((bad, good[fmt]()), (good[fmt](), bad)):
            with pytest.raises((ValueError, TypeError)):
                call(*pools, kv_format=fmt)
    with pytest.raises((ValueError, TypeError)):
        call(_bf16_pool(), _bf16_pool(), desc=_desc(num_blocks=BLOCKS + 1))
    assert len(lib.calls) == 6


def test_latent_pool(lib):
    desc = _desc(num_kv_heads=1, head_dim_qk=576, head_dim_v=512, latent=True)
    args = (Device(N, dtype=torch.int64), Device(BLOCKS, BS, 1, 576), None, Device(N, 1, 576), None)
    fnpu.kv_read(desc, *args, stream=0)
    small = Device(BLOCKS - 1, BS, 1, 576)
    for v in (None, small):  # (v_cache is not looked at)
        with pytest.raises((ValueError, TypeError)):
            fnpu.kv_read(desc, args[0], small, v, *args[3:], stream=0)
    assert len(lib.calls) == 1


def _plan(fmt, desc=None, n=N):
    return fnpu.Plan(0, desc or _desc(), n, fmt)


@pytest.mark.parametrize("fmt", [fnpu.KV_INT8_BLOCK, fnpu.KV_E4M3_BLOCK])
def test_runs_of_8_bit_plans_check_the_pools(lib, fmt):
    plan = _plan(fmt)
    q, lse, rows, slots = Device(N, HQ, D), Device(N, HQ, dtype=torch.float32), Device(N, HKV, D), Device(N, dtype=torch.int64)
    ok = _byte_pool()
    fnpu.mixed_attn_run(plan, q, ok, ok, q, lse, stream=0)
    fnpu.mixed_step(plan, rows, rows, slots, q, ok, ok, q, lse, stream=0)
    for bad in (_bf16_pool(), _byte_pool(BLOCKS * BLOCK - 1)):
        for pools in ((bad, ok), (ok, bad)):
            with pytest.raises((ValueError, TypeError)):
                fnpu.mixed_attn_run(plan, q, *pools, q, lse, stream=0)
            with pytest.raises((ValueError, TypeError)):
                fnpu.mixed_step(plan, rows, rows, slots, q, *pools, q, lse, stream=0)
    plan.desc.num_blocks = 1  # the plan's block ids are of the descriptor that it was made with
    with pytest.raises(ValueError):
        fnpu.mixed_attn_run(plan, q, _byte_pool(BLOCK), _byte_pool(BLOCK), q, lse, stream=0)
    assert [name for name, _ in lib.calls] == ["fnpu_mixed_attn_run", "fnpu_mixed_step"]


@pytest.fixture
def caches(monkeypatch):
    """Cache objects of three formats whose pools and outputs have no memory."""
    from paper_2606_04415_gb300.rotary import RotaryCache
    f = Device(D // 2, dtype=torch.float32)
    made = {fmt: RotaryCache(HQ, HKV, D, BS, BLOCKS, fnpu.make_rope(D), f, fmt, device="meta") for fmt, _ in GOOD}
    for fmt, pool in GOOD:
        made[fmt].k, made[fmt].v = pool(), pool()
    monkeypatch.setattr(RotaryCache, "_empty", lambda self, stream, *outputs: [Device(*s, dtype=t) for s, t in outputs])
    monkeypatch.setattr(fnpu, "_lib", Library())
    return made


def test_cache_refuses_another_caches_plan(caches):
    """A plan of another format or shape reads by other strides, and block ids of a larger
    pool lie past this one."""
    meta = (np.array([N]), np.array([N]), np.array([0]), np.zeros((1, 1), np.int32))
    q, calls = Device(N, HQ, D), fnpu._lib.calls
    for fmt, cache in caches.items():
        own = _plan(fmt)  # (another object of the same descriptor: layers share a plan)
        cache.attend(own, q, stream=0)
        cache.plan(*meta, plan=own, stream=0)
        done = len(calls)
        for bad in (_plan((fmt + 1) % 3), _plan((fmt + 2) % 3), _plan(fmt, _desc(num_blocks=BLOCKS + 1)), _plan(fmt, _desc(block_size=32)),
                    _plan(fmt, _desc(num_q_heads=8))):
            with pytest.raises(ValueError):
                cache.attend(bad, q, stream=0)
            with pytest.raises(ValueError):
                cache.plan(*meta, plan=bad, stream=0)
        assert len(calls) == done


def test_attend_refuses_other_queries(caches):
    """The planned rows are read from q and written to outputs of its size."""
    calls = fnpu._lib.calls
    for fmt, cache in caches.items():
        plan = _plan(fmt)
        for bad in (Device(N - 1, HQ, D), Device(N + 1, HQ, D), Device(N, HQ - 1, D), Device(N, HQ, D // 2), Device(N, HQ, D, dtype=torch.float16),
                    Device(N * HQ, D)):
            with pytest.raises((ValueError, TypeError)):
                cache.attend(plan, bad, stream=0)
        assert not calls


def test_one_token_has_no_stride(lib):
    """The stride between tokens means nothing where there is one; torch may report any."""
    one = [Device(1, h, D, stride=(s, D, 1), ptr=4096 * (i + 1)) for i, (h, s) in enumerate(((HQ, 301), (HKV, 1), (HKV, 129)))]
    fnpu.rope_append(_desc(), fnpu.make_rope(D), Device(D // 2, dtype=torch.float32), Device(1, 1, dtype=torch.int32), *one,
                     Device(1, dtype=torch.int64), Device(1, HQ, D, ptr=4096), _bf16_pool(), _bf16_pool(), stream=0)
    args = lib.calls[0][1]
    assert args[6] == HQ * D and args[8] == HKV * D and args[10] == HKV * D  # q (in place), keys, values
    x = Device(1, HQ, D, stride=(HQ * D + 9, D, 1))
    fnpu.rope(fnpu.make_rope(D), Device(D // 2, dtype=torch.float32), Device(1, 1, dtype=torch.int32), x, Device(1, HQ, D), stream=0)
    args = lib.calls[1][1]
    assert args[4] == args[9] == HQ * D


def test_raw_addresses_are_taken_as_they_are():
    """An integer is not asked for a tensor's attributes first (0.5 us each)."""
    class Address(int):
        def __getattr__(self, name):
            raise AssertionError(name)
    assert fnpu._dptr(Address(4096)) == 4096 and fnpu._dptr(None) is None
    assert fnpu._dptr(Device(3, ptr=64)) == 64
    for bad, error in ((Device(3, contiguous=False), ValueError), (torch.zeros(3), ValueError), ([1], TypeError), (4.0, TypeError)):
        with pytest.raises(error):
            fnpu._dptr(bad)
