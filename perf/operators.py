"""Measured cases of the rotary and 8-bit block-scaled cache operators.

Four paths, each a call or two that a serving program makes per layer:

* ``rope``: the rotation of packed rows [n, heads, d] by positions on one to
  three axes (``inverse``: the gradient of it).
* ``append``: ``rope_append`` of a step's rows -- the queries and new keys
  rotated, keys and values stored in the paged cache -- where the rows are
  slices of one fused projection's output. Over an 8-bit cache, ``kv_read``
  then reads the blocks that the step wrote to back as bf16.
* ``attend``: attention of a planned step over the 8-bit cache
  (``mixed_attn_run`` of a plan that all layers share).

The 8-bit cache: pools of blocks, a block holding codes [kv heads][slots][d]
and one fp32 scale, a power of two 2^e, for each kv head (padded to 16 bytes).
A stored value is (code - 128) 2^e (``int8``) or the e4m3 value of the code
times 2^e (``e4m3``); e is the least integer for which the block's largest
magnitude fits (127 or 448 times 2^e), between -60 and 60. An append to a
block that holds rows already keeps the larger exponent and stores those rows
anew where it grew.

Head shapes, block sizes and lengths are those of the repository's workloads
and tests. Queries are N(0, 4) before attention and N(0, 1) before a rotation,
cache rows N(0, s^2) with an s between 1/2 and 2 of each block and head, as
heads and stretches of text differ. Lengths depend on the case alone (``lens``
seeds them); values and the places of blocks in the pool on the seed.
"""
import math

import numpy as np
import torch

own = False

# (query heads, kv heads, width)
HEADS = {
    "4x2": (4, 2, 64),        # the small exhaustive-check shape
    "8x1": (8, 1, 64),        # one kv head
    "28x4": (28, 4, 128),     # Qwen2.5-7B
    "32x8": (32, 8, 128),     # R1-Distill-Llama-8B
}
FORMATS = ("bf16", "int8", "e4m3")
LARGEST = {"int8": 127.0, "e4m3": 448.0}
LEAST_E, MOST_E = -60, 60


def _rope(heads, d, n, axes, rot, interleaved=False, inverse=False, lens=0):
    return dict(path="rope", heads=heads, d=d, n=n, axes=axes, rot=rot, interleaved=interleaved, inverse=inverse, lens=lens)


def _step(path, heads, fmt, bs, chunks, chunk, prefix, decodes, ctx_lo, ctx_hi, tokens=1, axes=1, lens=0):
    """``chunks`` prefill chunks of ``chunk`` tokens on prefixes of up to
    ``prefix`` and ``decodes`` decodes of ``tokens`` tokens each with contexts
    of ``ctx_lo`` .. ``ctx_hi``."""
    return dict(path=path, heads=heads, fmt=fmt, bs=bs, chunks=chunks, chunk=chunk, prefix=prefix, decodes=decodes, ctx_lo=ctx_lo,
                ctx_hi=ctx_hi, tokens=tokens, axes=axes, lens=lens)


def listed():
    return [
        # the patches of one small image, height and width
        dict(_rope(16, 64, 256, 2, 64), name="rope_image"),
        # the queries of a video prompt, time, height and width
        dict(_rope(28, 128, 24000, 3, 128), name="rope_video"),
        # the gradient of a rotation of half of each head, neighbouring columns paired
        dict(_rope(32, 128, 3001, 1, 64, interleaved=True, inverse=True), name="rope_grad"),
        # a decode step's rows into a bf16 cache
        dict(_step("append", "28x4", "bf16", 16, 0, 0, 0, 64, 512, 4096), name="append_64"),
        # a long multi-modal prompt into a bf16 cache
        dict(_step("append", "32x8", "bf16", 32, 1, 8192, 0, 0, 0, 0, axes=3), name="append_8192"),
        # a decode step's rows into an 8-bit cache: one row a block, most blocks partly filled
        dict(_step("append", "28x4", "e4m3", 16, 0, 0, 0, 128, 128, 8192), name="append_128_e4m3"),
        # a prompt chunk into an 8-bit cache, from the middle of a block on
        dict(_step("append", "28x4", "int8", 16, 1, 2048, 7001, 0, 0, 0), name="append_2048_int8"),
        # a lightly loaded server: four decodes, a latency-bound call
        dict(_step("attend", "28x4", "int8", 16, 0, 0, 0, 4, 300, 2500), name="decode_4_int8"),
        # an ordinary decode batch, bound by cache reads
        dict(_step("attend", "28x4", "e4m3", 16, 0, 0, 0, 64, 512, 4096), name="decode_64_e4m3"),
        # a full server: the largest decode batch, blocks of 32
        dict(_step("attend", "32x8", "int8", 32, 0, 0, 0, 256, 500, 8000), name="decode_256_int8"),
        # prefill and decode co-located: one chunk on a long prefix beside 128 decodes
        dict(_step("attend", "28x4", "int8", 16, 1, 2048, 7000, 128, 128, 8192), name="mixed_2048_128_int8"),
        # speculative verification on long contexts: 16 sequences of four tokens each
        dict(_step("attend", "28x4", "e4m3", 64, 0, 0, 0, 16, 2000, 30000, tokens=4), name="verify_16x4_e4m3"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    lens = rng.randrange(1 << 20)
    kind = rng.choice(["rope", "rope", "append", "append", "append", "decode", "decode", "decode", "verify", "prefill", "mixed"])
    heads = rng.choice(["4x2", "8x1", "28x4", "28x4", "32x8", "32x8"])
    bs = rng.choice([16, 32, 64])
    if kind == "rope":
        h, d = rng.choice([4, 8, 12, 16, 28, 32]), rng.choice([64, 80, 128])
        return _rope(h, d, spread(1, 800000 // (h * d // 64)), rng.randint(1, 3), rng.choice([d, d // 2]), rng.random() < 0.4,
                     rng.random() < 0.4, lens)
    if kind == "append":
        fmt, axes = rng.choice(FORMATS), rng.choice([1, 1, 3])
        if rng.random() < 0.5:
            return _step("append", heads, fmt, bs, 0, 0, 0, spread(1, 256), 100, spread(200, 6000), rng.choice([1, 1, 4]), axes, lens)
        n = rng.randint(1, 4)
        return _step("append", heads, fmt, bs, n, spread(20, 8000 // n), spread(1, 4000), 0, 0, 0, 1, axes, lens)
    fmt = rng.choice(FORMATS[1:])
    lo = spread(20, 1000)
    if kind == "decode":
        n = spread(1, 200)
        return _step("attend", heads, fmt, bs, 0, 0, 0, n, lo, lo + spread(50, min(100000, 1600000 // n)), lens=lens)
    if kind == "verify":
        n = spread(1, 64)
        return _step("attend", heads, fmt, bs, 0, 0, 0, n, lo, lo + spread(50, min(30000, 300000 // n)), rng.randint(2, 8), lens=lens)
    n = rng.randint(1, 3)
    chunk, prefix = spread(20, 2000 // n), spread(1, 7000)
    if kind == "prefill":
        return _step("attend", heads, fmt, bs, n, chunk, prefix, 0, 0, 0, lens=lens)
    return _step("attend", heads, fmt, bs, n, chunk, prefix, spread(1, 130), lo, lo + spread(50, 7000), lens=lens)


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """(query_len, context_len, phase) of the case's sequences."""
    rng = np.random.default_rng([19, case["lens"]])
    n, dec = case["chunks"], case["decodes"]
    pre = [case["prefix"] * i // (n - 1) if n > 1 else case["prefix"] for i in range(n)]
    q = [case["chunk"]] * n + [case["tokens"]] * dec
    lo, hi = max(1, case["ctx_lo"]), max(1, case["ctx_hi"])
    drawn = np.exp(rng.uniform(math.log(lo), math.log(hi), dec)) if n else rng.uniform(lo, hi, dec)
    ctx = [case["chunk"] + p for p in pre] + [max(case["tokens"], int(c)) for c in drawn]
    return np.array(q, np.int32), np.array(ctx, np.int32), np.array([0] * n + [1] * dec, np.uint8)


def _block_bytes(hkv, bs, d):
    return hkv * bs * d + 16 * ((hkv + 3) // 4)


def _views(pool, blocks, hkv, bs, d):
    """Codes [blocks, hkv, bs, d] and scales [blocks, hkv] of an 8-bit pool."""
    b = _block_bytes(hkv, bs, d)
    codes = pool.as_strided((blocks, hkv, bs, d), (b, bs * d, d, 1))
    return codes, pool.view(torch.float32).as_strided((blocks, hkv), (b // 4, 1), hkv * bs * d // 4)


def _exponent(amax, fmt):
    """The least e with amax <= largest * 2^e, within the format's range."""
    m, x = torch.frexp(amax)
    e = x - 7 + (m > 127 / 128).to(x.dtype) if fmt == "int8" else x - 9 + (m > 448 / 512).to(x.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, LEAST_E)).clamp(LEAST_E, MOST_E)


def _encode(x, fmt):
    """Codes of values that the scale has been taken from."""
    if fmt == "int8":
        return (x.round().clamp(-127, 127) + 128).to(torch.uint8)
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(codes, fmt, dtype=torch.float32):
    return codes.to(dtype) - 128 if fmt == "int8" else codes.contiguous().view(torch.float8_e4m3fn).to(dtype)


def _positions(case, n, q_len, ctx):
    """Positions [axes, n], as a program lays them out: of tokens along their
    sequence, of patches over frames of a grid that is wider than high."""
    if case["path"] == "append":
        at = np.concatenate([np.arange(c - q, c) for q, c in zip(q_len, ctx)])
        if case["axes"] == 1:
            return at[None, :].astype(np.int32)
        start = np.concatenate([np.full(q, c - q) for q, c in zip(q_len, ctx)])
        i = at - start
        return np.stack([start + i // 1200, start + i // 40 % 30, start + i % 40]).astype(np.int32)
    i = np.arange(n)
    w = max(1, int(math.sqrt(n) * 1.3)) if case["axes"] == 2 else 40
    grid = [i // w, i % w] if case["axes"] == 2 else [i // 1200, i // 40 % 30, i % 40]
    return np.stack([i + 700] if case["axes"] == 1 else grid).astype(np.int32)


def _pair_axis(pairs, axes):
    """Axis of each pair: time takes a quarter, the others the rest in equal parts."""
    if axes == 3:
        cut = [pairs // 4, pairs // 4 + (pairs - pairs // 4) // 2]
        return np.searchsorted(cut, np.arange(pairs), side="right").astype(np.uint8)
    return (np.arange(pairs) * axes // pairs).astype(np.uint8)


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, std=1.0):
        return (torch.randn(shape, device="cuda", dtype=torch.float32, generator=g) * std).to(torch.bfloat16)

    x = {"case": dict(case)}
    if case["path"] == "rope":
        n, h, d, rot = case["n"], case["heads"], case["d"], case["rot"]
        pos = _positions(case, n, None, None)
        x["x"], x["out"] = normal(n, h, d), torch.empty((n, h, d), dtype=torch.bfloat16, device="cuda")
    else:
        hq, hkv, d = HEADS[case["heads"]]
        bs, rot = case["bs"], d
        q_len, ctx, phase = _lengths(case)
        T = int(q_len.sum())
        nblk = (ctx.astype(np.int64) + bs - 1) // bs
        blocks = int(math.ceil(1.25 * int(nblk.sum())))
        rng = np.random.default_rng([31, int(seed)])
        perm = rng.permutation(blocks).astype(np.int32)
        bt = rng.integers(0, blocks, size=(len(ctx), int(nblk.max()) + 1)).astype(np.int32)
        off = np.concatenate([[0], np.cumsum(nblk)])
        for s in range(len(ctx)):
            bt[s, :nblk[s]] = perm[off[s]:off[s + 1]]
        x.update(q_len=q_len, ctx=ctx, phase=phase, bt=bt, blocks=blocks, T=T)
        if case["path"] == "append":
            x["qkv"] = normal(T, hq + 2 * hkv, d)      # one projection's output: queries, keys, values
            new, rows, block_of, token_of, touched, at = [], [], [], [], [], 0
            for s in range(len(ctx)):
                p0, c = int(ctx[s] - q_len[s]), int(ctx[s])
                pos = np.arange(p0 // bs * bs, c, dtype=np.int64)   # the rows of the blocks written to
                sl = bt[s, pos // bs].astype(np.int64) * bs + pos % bs
                rows.append(sl)
                new.append(sl[pos >= p0])
                block_of.append(pos // bs - p0 // bs + sum(len(t) for t in touched))
                token_of.append(np.where(pos >= p0, at + pos - p0, -1))
                touched.append(bt[s, p0 // bs:(c + bs - 1) // bs].astype(np.int64))
                at += c - p0
            for key, v in (("slots", new), ("rows", rows), ("block_of", block_of), ("token_of", token_of), ("touched", touched)):
                x[key] = torch.from_numpy(np.concatenate(v)).cuda()
            x["q_out"] = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")
            pos = _positions(case, T, q_len, ctx)
        else:
            x["q"] = normal(T, hq, d, std=2.0)
            x["out"] = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")
            x["lse"] = torch.empty((T, hq), dtype=torch.float32, device="cuda")
            x["bt_dev"], x["ctx_dev"], x["q_dev"] = (torch.from_numpy(a.astype(np.int64)).cuda() for a in (bt, ctx, q_len))
        for name in ("k", "v"):
            if case["fmt"] == "bf16":
                x[name] = normal(blocks, bs, hkv, d)
                continue
            pool = torch.zeros(blocks * _block_bytes(hkv, bs, d), dtype=torch.uint8, device="cuda")
            codes, scales = _views(pool, blocks, hkv, bs, d)
            for i in range(0, blocks, 1 << 14):
                n = min(blocks - i, 1 << 14)
                f = torch.randn((n, hkv, bs, d), device="cuda", generator=g)
                f *= torch.exp2(torch.rand((n, hkv, 1, 1), device="cuda", generator=g) * 2 - 1)
                e = _exponent(f.abs().amax((2, 3)), case["fmt"])
                codes[i:i + n] = _encode(f * torch.exp2(-e.float())[:, :, None, None], case["fmt"])
                scales[i:i + n] = torch.exp2(e.float())
            x[name] = pool
        if case["path"] == "append" and case["fmt"] != "bf16":
            x["k_rows"], x["v_rows"] = (torch.empty((x["rows"].numel(), hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if case["path"] != "attend":
        x["pair_axis"] = _pair_axis(rot // 2, case["axes"])
        x["axis_dev"] = torch.from_numpy(x["pair_axis"].astype(np.int64)).cuda()
        x["positions"] = torch.from_numpy(pos).cuda()
        base = 1e6 if case["axes"] == 3 else 1e4
        x["inv_freq"] = torch.from_numpy((base ** (-np.arange(rot // 2) * 2.0 / rot)).astype(np.float32)).cuda()
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    if own:  # the descriptors and the plan that a program keeps
        import paper_2606_04415_gb300 as fnpu
        x["fnpu"] = fnpu
        if case["path"] != "attend":
            x["rope"] = fnpu.make_rope(2 * len(x["pair_axis"]), interleaved=case.get("interleaved", False),
                                       inverse=case.get("inverse", False), num_axes=case["axes"], pair_axis=x["pair_axis"])
        if case["path"] != "rope":
            hq, hkv, d = HEADS[case["heads"]]
            x["desc"] = fnpu.make_desc(hq, hkv, d, d, case["bs"], x["blocks"])
            x["fmt"] = {"bf16": fnpu.KV_BF16, "int8": fnpu.KV_INT8_BLOCK, "e4m3": fnpu.KV_E4M3_BLOCK}[case["fmt"]]
        if case["path"] == "attend":
            x["plan"] = fnpu.kv8_attn_plan(x["desc"], x["fmt"], x["q_len"], x["ctx"], x["phase"], x["bt"])
    return x


# --------------------------------------------------------------- plain form

def _rotate(f, x, interleaved=False, inverse=False):
    """fp32 rows [n, heads, d] with their first 2 * pairs columns rotated."""
    pairs = x["inv_freq"].numel()
    angle = x["positions"][x["axis_dev"]].T.float() * x["inv_freq"]
    c, s = torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]
    s = -s if inverse else s
    a, b = (f[..., 0:2 * pairs:2], f[..., 1:2 * pairs:2]) if interleaved else (f[..., :pairs], f[..., pairs:2 * pairs])
    y = [a * c - b * s, b * c + a * s]
    y = torch.stack(y, -1).flatten(-2) if interleaved else torch.cat(y, -1)
    return torch.cat([y, f[..., 2 * pairs:]], -1)


def _store(pool, new, x):
    """New fp32 rows into an 8-bit pool; the rows of the blocks written to."""
    case = x["case"]
    hq, hkv, d = HEADS[case["heads"]]
    bs, fmt = case["bs"], case["fmt"]
    codes, scales = _views(pool, x["blocks"], hkv, bs, d)
    block, slot, at, token = x["rows"] // bs, x["rows"] % bs, x["block_of"], x["token_of"]
    fresh = (token >= 0)[:, None, None]
    f = torch.where(fresh, new[token.clamp(min=0)], _decode(codes[block, :, slot], fmt) * scales[block][..., None])
    zero = torch.zeros((x["touched"].numel(), hkv), device=new.device)
    amax = zero.index_reduce(0, at, torch.where(fresh, f, torch.zeros_like(f)).abs().amax(-1), "amax")
    # (the exponent so far of the blocks that hold rows already)
    held = zero[:, 0].index_reduce(0, at, (token < 0).float(), "amax") > 0
    before = torch.where(held[:, None], torch.frexp(scales[x["touched"]])[1] - 1, torch.full_like(zero, LEAST_E, dtype=torch.int32))
    e = torch.maximum(_exponent(amax, fmt), before).float()
    c = _encode(f * torch.exp2(-e)[at][..., None], fmt)
    codes[block, :, slot] = c
    scales[x["touched"]] = torch.exp2(e)
    return (_decode(c, fmt) * torch.exp2(e)[at][..., None]).to(torch.bfloat16)


def _attend(x, first, last, t0, t1, out, lse):
    """Attention of the sequences first .. last - 1, all of the same number of
    tokens (t0 .. t1 - 1 of the step), padded to the longest context."""
    case = x["case"]
    hq, hkv, d = HEADS[case["heads"]]
    bs, n = case["bs"], last - first
    if n == 0:
        return
    q = x["q"][t0:t1].float().view(n, -1, hkv, hq // hkv, d)
    ctx = x["ctx_dev"][first:last]
    nb = int((x["ctx"][first:last].max() + bs - 1) // bs)
    table = x["bt_dev"][first:last, :nb]
    keys = torch.arange(nb * bs, device=q.device)

    def rows(pool):
        codes, scales = _views(pool, x["blocks"], hkv, bs, d)
        f = _decode(codes[table], case["fmt"]) * scales[table][..., None, None]
        # (columns of the table past a sequence's blocks name blocks that are not its own)
        f = f.permute(0, 2, 1, 3, 4).reshape(n, hkv, nb * bs, d)
        return torch.where((keys < ctx[:, None])[:, None, :, None], f, torch.zeros((), device=f.device))

    pos = ctx[:, None] - q.shape[1] + torch.arange(q.shape[1], device=q.device)
    s = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d), rows(x["k"]).transpose(2, 3)).view(n, hkv, q.shape[1], hq // hkv, -1)
    s = s * d ** -0.5
    s = torch.where((keys <= pos[:, :, None])[:, None, :, None, :], s, torch.full((), -math.inf, device=s.device))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul((p / z).view(n, hkv, -1, nb * bs), rows(x["v"])).view(n, hkv, q.shape[1], hq // hkv, d)
    out[t0:t1] = o.permute(0, 2, 1, 3, 4).reshape(t1 - t0, hq, d).to(torch.bfloat16)
    lse[t0:t1] = (m + torch.log(z))[..., 0].permute(0, 2, 1, 3).reshape(t1 - t0, hq)


def run(x):
    case = x["case"]
    if case["path"] == "rope":
        if own:
            x["fnpu"].rope(x["rope"], x["inv_freq"], x["positions"], x["x"], x["out"])
            return {"out": x["out"]}
        return {"out": _rotate(x["x"].float(), x, case["interleaved"], case["inverse"]).to(torch.bfloat16)}
    hq, hkv, d = HEADS[case["heads"]]
    if case["path"] == "attend":
        if own:
            x["fnpu"].mixed_attn_run(x["plan"], x["q"], x["k"], x["v"], x["out"], x["lse"])
        else:
            n, t = case["chunks"], case["chunks"] * case["chunk"]
            _attend(x, 0, n, 0, t, x["out"], x["lse"])
            _attend(x, n, n + case["decodes"], t, x["T"], x["out"], x["lse"])
        return {"out": x["out"], "lse": x["lse"]}
    q, k, v = x["qkv"][:, :hq], x["qkv"][:, hq:hq + hkv], x["qkv"][:, hq + hkv:]
    if own:
        x["fnpu"].rope_append(x["desc"], x["rope"], x["inv_freq"], x["positions"], q, k, v, x["slots"], x["q_out"], x["k"], x["v"],
                              kv_format=x["fmt"])
        if case["fmt"] != "bf16":
            x["fnpu"].kv_read(x["desc"], x["rows"], x["k"], x["v"], x["k_rows"], x["v_rows"], kv_format=x["fmt"])
            return {"q": x["q_out"], "k": x["k_rows"], "v": x["v_rows"]}
        return {"q": x["q_out"], "k": x["k"], "v": x["v"]}
    qr, kr = _rotate(q.float(), x).to(torch.bfloat16), _rotate(k.float(), x)
    if case["fmt"] != "bf16":
        return {"q": qr, "k": _store(x["k"], kr, x), "v": _store(x["v"], v.float(), x)}
    x["k"].view(-1, hkv, d)[x["slots"]] = kr.to(torch.bfloat16)
    x["v"].view(-1, hkv, d)[x["slots"]] = v
    return {"q": qr, "k": x["k"], "v": x["v"]}


# -------------------------------------------------------------------- work

def work(case):
    if case["path"] == "rope":
        n, h = case["n"], case["heads"]
        # rows read and written, positions
        return {"bytes": n * (4 * h * case["d"] + 4 * case["axes"]), "flops": n * h * 3 * case["rot"]}
    hq, hkv, d = HEADS[case["heads"]]
    q, ctx, _ = (a.astype(np.int64) for a in _lengths(case))
    bs, T, pre = case["bs"], int(q.sum()), ctx - q
    if case["path"] == "append":
        # the projection's rows read, queries written, positions and slots
        b = T * (2 * d * (2 * hq + 2 * hkv) + 4 * case["axes"] + 8)
        if case["fmt"] == "bf16":
            b += T * 4 * hkv * d
        else:  # codes of the new rows and scales stored, the written blocks' rows read back as bf16
            rows, blocks = int((ctx - pre // bs * bs).sum()), int(((ctx + bs - 1) // bs - pre // bs).sum())
            b += T * 2 * hkv * d + 16 * blocks * hkv + rows * (8 + 6 * hkv * d)
        return {"bytes": b, "flops": T * (hq + hkv) * 3 * d}
    pairs = int((q * pre + q * (q + 1) // 2).sum())
    blocks = int(((ctx + bs - 1) // bs).sum())
    # every cached row's codes once, the blocks' scales, the table; queries, outputs
    return {"bytes": int(ctx.sum()) * 2 * hkv * d + blocks * (8 * hkv + 4) + T * hq * (4 * d + 4), "flops": 4 * hq * d * pairs}


# ------------------------------------------------------- the same in 64 bits

def _turned64(rows, x, interleaved=False, inverse=False):
    """Rows as complex numbers, multiplied by exp(i angle)."""
    f = rows.double().clone()
    n = x["inv_freq"].numel()
    axis = torch.from_numpy(x["pair_axis"].astype(np.int64)).to(f.device)
    angle = x["positions"].double()[axis, :].T * x["inv_freq"].double()
    turn = torch.polar(torch.ones_like(angle), -angle if inverse else angle)[:, None, :]
    one, two = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    z = torch.complex(f[..., one], f[..., two]) * turn
    f[..., one], f[..., two] = z.real, z.imag
    return f


def _fit64(top, fmt):
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / LARGEST[fmt]))
    e = e - (top <= LARGEST[fmt] * torch.exp2(e - 1)).double() + (top > LARGEST[fmt] * torch.exp2(e)).double()
    return e.clamp(LEAST_E, MOST_E)


def _near64(f, fmt):
    """The nearest value of the format to each (scaled) value, ties to even."""
    if fmt == "int8":
        return f.round().clamp(-127, 127)
    e = torch.floor(torch.log2(f.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return ((f / step).round() * step).clamp(-448, 448)


def _value64(codes, fmt):
    if fmt == "int8":
        return codes.double() - 128
    c = codes.long()
    e, m = c // 8 % 16, (c % 8).double()
    v = torch.where(e > 0, (8 + m) * torch.exp2(e.double() - 10), m * 2.0 ** -9)
    return torch.where(c > 127, -v, v)


def _stored64(x, pool, new):
    """The rows of the blocks that a step writes to, after it."""
    case = x["case"]
    hq, hkv, d = HEADS[case["heads"]]
    bs, fmt, blocks = case["bs"], case["fmt"], x["blocks"]
    raw = pool.view(blocks, -1)
    out, at = [], 0
    for s in range(len(x["ctx"])):
        p0, c = int(x["ctx"][s] - x["q_len"][s]), int(x["ctx"][s])
        ids = torch.from_numpy(x["bt"][s, p0 // bs:(c + bs - 1) // bs].astype(np.int64)).to(pool.device)
        n, lead = len(ids), p0 % bs
        grid = torch.zeros((n * bs, hkv, d), dtype=torch.float64, device=pool.device)
        grid[lead:lead + c - p0] = new[at:at + c - p0]
        grid = grid.view(n, bs, hkv, d)
        e = _fit64(grid.abs().amax((1, 3)), fmt)
        if lead:
            first = raw[int(ids[0])]
            e0 = torch.log2(first[hkv * bs * d:hkv * bs * d + 4 * hkv].clone().view(torch.float32).double()).round()
            old = _value64(first[:hkv * bs * d].view(hkv, bs, d), fmt) * torch.exp2(e0)[:, None, None]
            grid[0, :lead] = old.transpose(0, 1)[:lead]
            e[0] = torch.maximum(e[0], e0)
        unit = torch.exp2(e)[:, None, :, None]
        out.append((_near64(grid / unit, fmt) * unit).view(n * bs, hkv, d)[:lead + c - p0])
        at += c - p0
    return torch.cat(out)


def exact(case, seed):
    x = _inputs(case, seed)
    if case["path"] == "rope":
        return {"out": _turned64(x["x"], x, case["interleaved"], case["inverse"])}
    hq, hkv, d = HEADS[case["heads"]]
    bs, fmt = case["bs"], case["fmt"]
    if case["path"] == "append":
        f = x["qkv"].double()
        r = {"q": _turned64(f[:, :hq], x), "k": _turned64(f[:, hq:hq + hkv], x), "v": f[:, hq + hkv:]}
        for name in ("k", "v"):
            if fmt != "bf16":
                r[name] = _stored64(x, x[name], r[name])
            else:
                c = x[name].double().view(-1, hkv, d)
                c[x["slots"]] = r[name]
                r[name] = c.view(x[name].shape)
        return r
    G, blocks, b, at, outs, lses = hq // hkv, x["blocks"], hkv * bs * d, 0, [], []
    for s in range(len(x["ctx"])):
        n, c = int(x["q_len"][s]), int(x["ctx"][s])
        ids = torch.from_numpy(x["bt"][s, :(c + bs - 1) // bs].astype(np.int64)).cuda()
        kv = []
        for name in ("k", "v"):
            raw = x[name].view(blocks, -1)[ids]
            unit = raw[:, b:b + 4 * hkv].contiguous().view(torch.float32).double()
            kv.append((_value64(raw[:, :b].view(len(ids), hkv, bs, d), fmt) * unit[:, :, None, None]).transpose(0, 1).reshape(hkv, -1, d)[:, :c])
        q = x["q"][at:at + n].double()
        at += n
        o, l = torch.empty((n, hq, d), dtype=torch.float64, device="cuda"), torch.empty((n, hq), dtype=torch.float64, device="cuda")
        hidden = torch.arange(c, device="cuda")[None, :] > torch.arange(c - n, c, device="cuda")[:, None]
        step = max(1, (1 << 28) // max(1, c * G))
        for h in range(hkv):
            for i in range(0, n, step):
                qi = q[i:i + step, h * G:(h + 1) * G]
                sc = torch.einsum("ngd,cd->ngc", qi, kv[0][h]) / math.sqrt(d)
                sc = sc.masked_fill(hidden[i:i + step, None, :], -math.inf)
                le = torch.logsumexp(sc, -1)
                o[i:i + step, h * G:(h + 1) * G] = torch.einsum("ngc,cd->ngd", torch.exp(sc - le[..., None]), kv[1][h])
                l[i:i + step, h * G:(h + 1) * G] = le
        outs.append(o)
        lses.append(l)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
