"""Measured cases of windowed attention, beam selection and the pages of a cache.

Five paths, each a call or a few that a serving program makes in a step:

* ``step``: attention of a planned step (``window_attn_plan``, then
  ``mixed_attn_run``) in which a query at position p sees keys p - window + 1
  .. p and the first ``sinks`` keys of its sequence.
* ``rows``: the same for one token a sequence, with lengths and block table on
  the device and no plan (``window_decode``).
* ``beam``: the best continuations of every group of beams (``beam_select``):
  over beams b and tokens v, score[b] + log softmax(logits[b])[v], best first,
  ties to the lowest b, then v; b is given as a row of all groups' beams. A finished beam continues with the end token
  alone, at its own score; logits of -inf are no candidates.
* ``turn``: what a beam step does to the pages of a cache: those behind the
  window are freed (``pages_free``), the rows continue the beams chosen by
  ``parents``, each with room for its next tokens (``pages_fork``), and the
  partly filled pages that several rows would write to are copied
  (``kv_copy_blocks``, all layers in one call).
* ``compact``: live pages move to the lowest places of the pool
  (``pages_compact``, then ``kv_copy_blocks``).

A row of a block table holds the ids of its pages, column j for positions j *
bs on; -1 stands for a page that was freed. ``refs`` counts the places that
hold a page; a page without any is free, and new ones are the lowest free ids
in the order of the rows.

Head shapes, block sizes and lengths are those of the repository's workloads
and tests, vocabularies generic. Queries are N(0, 4), cache rows and logits
N(0, 1) and N(0, 6). Lengths depend on the case alone (``lens`` seeds them);
values and the places of blocks in the pool on the seed.
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


def _attn(path, heads, bs, window, sinks, chunks, chunk, prefix, decodes, ctx_lo, ctx_hi, tokens=1, lens=0):
    """``chunks`` prefill chunks of ``chunk`` tokens on prefixes of up to
    ``prefix`` and ``decodes`` decodes of ``tokens`` tokens each with contexts
    of ``ctx_lo`` .. ``ctx_hi``."""
    return dict(path=path, heads=heads, bs=bs, window=window, sinks=sinks, chunks=chunks, chunk=chunk, prefix=prefix, decodes=decodes,
                ctx_lo=ctx_lo, ctx_hi=ctx_hi, tokens=tokens, lens=lens)


def _beam(groups, beams, vocab, select, dtype, lens=0):
    return dict(path="beam", groups=groups, beams=beams, vocab=vocab, select=select, dtype=dtype, lens=lens)


def _pages(path, heads, bs, layers, groups, beams, ctx_lo, ctx_hi, window=0, sinks=0, grow=1, spare=0.25, lens=0):
    """``groups`` prompts of ``beams`` rows each that share their first pages;
    ``spare``: free pages of the pool, as a share of the live ones."""
    return dict(path=path, heads=heads, bs=bs, layers=layers, groups=groups, beams=beams, ctx_lo=ctx_lo, ctx_hi=ctx_hi, window=window,
                sinks=sinks, grow=grow, spare=spare, lens=lens)


def listed():
    return [
        # a lightly loaded server: four sequences, a latency-bound call
        dict(_attn("rows", "28x4", 16, 1024, 4, 0, 0, 0, 4, 300, 2500), name="rows_4"),
        # a full server on long texts, most of their pages freed
        dict(_attn("rows", "32x8", 16, 4096, 4, 0, 0, 0, 128, 2000, 60000), name="rows_128"),
        # an ordinary planned decode batch, some texts shorter than the window
        dict(_attn("step", "28x4", 16, 2048, 16, 0, 0, 0, 64, 512, 8192), name="step_decode_64"),
        # a long prompt in one piece, window alone
        dict(_attn("step", "32x8", 32, 2048, 0, 1, 8192, 0, 0, 0, 0), name="step_prompt_8192"),
        # prefill and decode co-located: one chunk on a long prefix beside 128 decodes
        dict(_attn("step", "28x4", 16, 4096, 4, 1, 2048, 7000, 128, 128, 8192), name="step_mixed_2048_128"),
        # one request of four beams
        dict(_beam(1, 4, 32000, 8, "bf16"), name="beam_1x4"),
        # fp32 logits over an odd vocabulary, rows that start anywhere
        dict(_beam(16, 5, 50257, 10, "fp32"), name="beam_16x5_fp32"),
        # a full server of eight beams a request
        dict(_beam(64, 8, 151936, 16, "bf16"), name="beam_64x8"),
        # two requests of four beams
        dict(_pages("turn", "28x4", 16, 2, 2, 4, 300, 2500, 1024, 4), name="turn_2x4"),
        # a full server of eight beams a request
        dict(_pages("turn", "28x4", 16, 4, 64, 8, 500, 8000, 2048, 4), name="turn_64x8"),
        # a small cache after some requests have left
        dict(_pages("compact", "32x8", 32, 2, 4, 4, 200, 1500, spare=0.5), name="compact_small"),
        # a large one
        dict(_pages("compact", "28x4", 16, 2, 64, 4, 500, 8000, spare=0.5), name="compact_large"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    lens = rng.randrange(1 << 20)
    kind = rng.choice(["rows", "rows", "decode", "verify", "prefill", "mixed", "beam", "beam", "beam", "turn", "turn", "compact"])
    heads = rng.choice(["4x2", "8x1", "28x4", "28x4", "32x8", "32x8"])
    bs = rng.choice([16, 32, 64])
    if kind == "beam":
        beams, vocab = spread(1, 16), spread(1000, 160000)
        return _beam(spread(1, max(1, min(64, 70000000 // (beams * vocab)))), beams, vocab, min(32, max(1, beams * rng.choice([1, 2, 2]))),
                     rng.choice(["bf16", "bf16", "fp32"]), lens)
    window, sinks, lo = spread(16, 5000), rng.choice([0, 1, 4, 16, 100]), spread(20, 1000)
    if kind in ("turn", "compact"):
        groups, beams = spread(1, 64), rng.randint(1, 8)
        hi = lo + spread(50, 7000)
        if kind == "turn":
            return _pages("turn", heads, bs, rng.randint(1, 4), groups, beams, lo, hi, rng.choice([0, window]), sinks, rng.choice([1, 1, 4]),
                          rng.choice([0.1, 0.5]), lens)
        return _pages("compact", heads, bs, rng.randint(1, 2), groups, min(beams, 4), lo, hi, spare=rng.choice([0.1, 0.5, 2.0]), lens=lens)
    if kind in ("rows", "decode"):
        n = spread(1, 200)
        return _attn("rows" if kind == "rows" else "step", heads, bs, window, sinks, 0, 0, 0, n, lo, lo + spread(50, 60000), lens=lens)
    if kind == "verify":
        return _attn("step", heads, bs, window, sinks, 0, 0, 0, spread(1, 64), lo, lo + spread(50, 30000), rng.randint(2, 8), lens)
    n = rng.randint(1, 3)
    chunk, prefix = spread(20, (8000 if kind == "prefill" else 2000) // n), spread(1, 7000)
    if kind == "prefill":
        return _attn("step", heads, bs, window, sinks, n, chunk, prefix, 0, 0, 0, lens=lens)
    return _attn("step", heads, bs, window, sinks, n, chunk, prefix, spread(1, 130), lo, lo + spread(50, 7000), lens=lens)


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """(query_len, context_len, phase) of the case's sequences."""
    rng = np.random.default_rng([23, case["lens"]])
    n, dec = case["chunks"], case["decodes"]
    pre = [case["prefix"] * i // (n - 1) if n > 1 else case["prefix"] for i in range(n)]
    q = [case["chunk"]] * n + [case["tokens"]] * dec
    lo, hi = max(1, case["ctx_lo"]), max(1, case["ctx_hi"])
    drawn = np.exp(rng.uniform(math.log(lo), math.log(hi), dec)) if n else rng.uniform(lo, hi, dec)
    ctx = [case["chunk"] + p for p in pre] + [max(case["tokens"], int(c)) for c in drawn]
    return np.array(q, np.int32), np.array(ctx, np.int32), np.array([0] * n + [1] * dec, np.uint8)


def _needed(held, first_open, sinks, bs):
    """Which of ``held`` columns hold a key below ``sinks`` or from ``first_open`` on."""
    col = np.arange(held)
    return (col * bs < sinks) | ((col + 1) * bs > first_open)


def _pages_of(case):
    """Rows that share pages: (lengths, pages of each row as numbers from 0, -1
    for those behind the window, and how many numbers there are)."""
    rng = np.random.default_rng([29, case["lens"]])
    bs, rows, length, count = case["bs"], [], [], 0
    for g in range(case["groups"]):
        n = int(rng.integers(case["ctx_lo"], case["ctx_hi"] + 1))
        held = (n + bs - 1) // bs
        alone = rng.integers(held // 2, held, case["beams"]) if held > 1 else np.zeros(case["beams"], np.int64)
        # (as the step before left it: freed for a sequence of one token less)
        live = _needed(held, n - case["window"], case["sinks"], bs) if case["window"] else np.ones(held, bool)
        # a chain of rows: each follows the one before up to its own place
        row = np.full(held, -1, np.int64)
        for b in range(case["beams"]):
            fresh = live & (np.arange(held) >= (alone[b] if b else 0))
            row = np.where(fresh, count + np.cumsum(fresh) - 1, row)
            count += int(fresh.sum())
            rows.append(row.copy())
            length.append(n)
    return np.array(length, np.int32), rows, count


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = np.random.default_rng([37, int(seed)])
    x = {"case": dict(case)}

    def normal(*shape, std=1.0):
        return (torch.randn(shape, device="cuda", dtype=torch.float32, generator=g) * std).to(torch.bfloat16)

    if case["path"] == "beam":
        b, w, v, k = case["groups"], case["beams"], case["vocab"], case["select"]
        x["logits"] = torch.randn((b, w, v), device="cuda", generator=g).mul_(math.sqrt(6.0))
        if case["dtype"] == "bf16":
            x["logits"] = x["logits"].to(torch.bfloat16)
        x["logits"][..., torch.from_numpy(rng.integers(0, v, v // 50)).cuda()] = -math.inf   # tokens that are ruled out
        x["scores"] = -20 * torch.rand((b, w), device="cuda", generator=g)
        x["finished"] = (torch.rand((b, w), device="cuda", generator=g) < 0.1).to(torch.uint8)
        x["out_scores"] = torch.empty((b, k), device="cuda")
        x["out_parents"], x["out_tokens"] = (torch.empty((b, k), dtype=torch.int32, device="cuda") for _ in range(2))
        return x
    hq, hkv, d = HEADS[case["heads"]]
    bs = case["bs"]
    if case["path"] in ("step", "rows"):
        q_len, ctx, phase = _lengths(case)
        T, held = int(q_len.sum()), (ctx.astype(np.int64) + bs - 1) // bs
        need = [_needed(int(held[s]), int(ctx[s] - q_len[s]) - case["window"] + 1, case["sinks"], bs) for s in range(len(ctx))]
        total = sum(int(n.sum()) for n in need)
        blocks = int(math.ceil(1.25 * total))
        perm, at = rng.permutation(blocks).astype(np.int32), 0
        bt = np.full((len(ctx), int(held.max()) + 1), -1, np.int32)   # pages behind the window: freed
        for s, n in enumerate(need):
            cols = np.flatnonzero(n)
            bt[s, cols] = perm[at:at + len(cols)]
            at += len(cols)
        x.update(q_len=q_len, ctx=ctx, phase=phase, bt=bt, blocks=blocks, T=T)
        x["q"] = normal(T, hq, d, std=2.0)
        x["k"], x["v"] = normal(blocks, bs, hkv, d), normal(blocks, bs, hkv, d)
        x["out"], x["lse"] = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((T, hq), device="cuda")
        x["bt_dev"], x["ctx_dev"] = torch.from_numpy(bt).cuda(), torch.from_numpy(ctx).cuda()
        return x
    length, rows, count = _pages_of(case)
    blocks = int(math.ceil(count * (1 + case["spare"]))) + case["groups"] * case["beams"] * (1 + case["grow"])
    perm = rng.permutation(blocks).astype(np.int32)
    R, width = len(rows), max(len(r) for r in rows) + 1 + (case["grow"] + bs - 1) // bs
    table = np.full((R, width), -1, np.int32)
    for r, row in enumerate(rows):
        table[r, :len(row)] = np.where(row >= 0, perm[row.clip(min=0)], -1)
    refs = np.bincount(table[table >= 0], minlength=blocks).astype(np.int32)
    # table, lengths and counts in one buffer, which a pass takes a copy of
    x["state"] = torch.from_numpy(np.concatenate([table.reshape(-1), length, refs])).cuda()
    x.update(R=R, width=width, blocks=blocks)
    if case["path"] == "turn":   # each beam of a request follows one of its beams
        group = np.arange(R) // case["beams"] * case["beams"]
        x["parents"] = torch.from_numpy((group + rng.integers(0, case["beams"], R)).astype(np.int32)).cuda()
    x["k"], x["v"] = ([normal(blocks, bs, hkv, d) for _ in range(case["layers"])] for _ in range(2))
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    if own:  # the descriptors, workspaces and the plan that a program keeps
        import paper_2606_04415_gb300 as fnpu
        x["fnpu"] = fnpu
        if case["path"] == "beam":
            n = fnpu.beam_select_workspace(case["groups"], case["beams"], case["vocab"], case["select"])
            x["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
            return x
        hq, hkv, d = HEADS[case["heads"]]
        x["desc"] = fnpu.make_desc(hq, hkv, d, d, case["bs"], x["blocks"])
        if case["path"] == "step":
            x["plan"] = fnpu.window_attn_plan(x["desc"], case["window"], case["sinks"], x["q_len"], x["ctx"], x["phase"], x["bt"])
        elif case["path"] == "rows":
            x["most"] = int(x["ctx"].max())
            n = fnpu.window_decode_workspace(x["desc"], case["window"], case["sinks"], len(x["ctx"]), x["most"])
            x["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        else:
            x["pages"] = fnpu.make_pages(case["bs"], x["blocks"])
            x["workspace"] = torch.empty(fnpu.pages_workspace(x["pages"], x["R"]), dtype=torch.uint8, device="cuda")
    return x


# --------------------------------------------------------------- plain form

def _attend(x, first, last, t0, t1, out, lse):
    """Attention of the sequences first .. last - 1, all of the same number of
    tokens (t0 .. t1 - 1 of the step): the sinks, then the keys from the first
    query's window on, padded to the longest."""
    case = x["case"]
    hq, hkv, d = HEADS[case["heads"]]
    bs, n, w, s = case["bs"], last - first, case["window"], case["sinks"]
    if n == 0:
        return
    q = x["q"][t0:t1].float().view(n, -1, hkv, hq // hkv, d)
    t = q.shape[1]
    ctx = x["ctx_dev"][first:last].long()[:, None]
    reach = min(t + w - 1, int(x["ctx"][first:last].max()))
    near = ctx - reach + torch.arange(reach, device=q.device)
    at = torch.cat([torch.arange(s, device=q.device).expand(n, s), near], 1)
    there = torch.cat([torch.arange(s, device=q.device) < ctx, near >= s], 1)
    page = torch.gather(x["bt_dev"][first:last].long(), 1, (at.clamp(min=0) // bs).clamp(max=x["bt_dev"].shape[1] - 1))
    there = there & (page >= 0)
    slot = torch.where(there, page * bs + at % bs, torch.zeros((), dtype=torch.long, device=q.device))

    def rows(pool):
        f = pool.view(-1, hkv, d)[slot].float().permute(0, 2, 1, 3)
        return torch.where(there[:, None, :, None], f, torch.zeros((), device=f.device))

    pos = ctx - t + torch.arange(t, device=q.device)
    seen = there[:, None, :] & (at[:, None, :] <= pos[:, :, None]) & ((at[:, None, :] > pos[:, :, None] - w) | (at < s)[:, None, :])
    a = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d), rows(x["k"]).transpose(2, 3)).view(n, hkv, t, hq // hkv, -1) * d ** -0.5
    a = torch.where(seen[:, None, :, None, :], a, torch.full((), -math.inf, device=a.device))
    m = a.amax(-1, keepdim=True)
    p = torch.exp(a - m)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul((p / z).view(n, hkv, t * (hq // hkv), -1), rows(x["v"])).view(n, hkv, t, hq // hkv, d)
    out[t0:t1] = o.permute(0, 2, 1, 3, 4).reshape(t1 - t0, hq, d).to(torch.bfloat16)
    lse[t0:t1] = (m + torch.log(z))[..., 0].permute(0, 2, 1, 3).reshape(t1 - t0, hq)


def _select(x):
    """In 64 bits: candidates of different beams may lie next to each other."""
    case = x["case"]
    f = x["logits"].double()
    m = f.amax(-1, keepdim=True)
    total = x["scores"].double()[..., None] + (f - m) - torch.log(torch.exp(f - m).sum(-1, keepdim=True))
    # a finished beam goes on with the end token alone
    end = (torch.arange(f.shape[2], device=f.device) == END) & (x["finished"] > 0)[..., None]
    total = torch.where((x["finished"] > 0)[..., None], torch.full((), -math.inf, dtype=f.dtype, device=f.device), total)
    total = torch.where(end, x["scores"].double()[..., None], total).flatten(1)
    best, at = torch.sort(total, dim=1, descending=True, stable=True)
    best, at = best[:, :case["select"]], at[:, :case["select"]]
    none = best == -math.inf
    beam = at // f.shape[2] + f.shape[1] * torch.arange(len(at), device=f.device)[:, None]   # as a row of all groups' beams
    parent, token = (torch.where(none, torch.full_like(at, -1), v).to(torch.int32) for v in (beam, at % f.shape[2]))
    return {"scores": best.float(), "parents": parent, "tokens": token}


END = 2  # the end token


def _views(x, state):
    n = x["R"] * x["width"]
    return state[:n].view(x["R"], x["width"]), state[n:n + x["R"]], state[n + x["R"]:]


def _count(refs, pages, by):
    """Counts of the pages (those below zero left out) changed by ``by``."""
    flat = pages.reshape(-1).long()
    refs.index_add_(0, flat.clamp(min=0), torch.where(flat >= 0, by, 0).to(refs.dtype))


def _turn(x, table, length, refs):
    case, bs, blocks, R, width = x["case"], x["case"]["bs"], x["blocks"], x["R"], x["width"]
    col = torch.arange(width, device=table.device)
    if case["window"]:  # pages that the next token does not see
        dead = (col * bs >= case["sinks"]) & ((col + 1) * bs <= (length + 1 - case["window"])[:, None]) & (table >= 0)
        _count(refs, torch.where(dead, table, torch.full_like(table, -1)), -1)
        table[dead] = -1
    parent, grow = x["parents"].long(), case["grow"]
    n = length[parent].long()
    held = (n + bs - 1) // bs
    new = torch.where(col < held[:, None], table[parent], torch.full_like(table, -1))
    _count(refs, torch.where(col < ((length.long() + bs - 1) // bs)[:, None], table, torch.full_like(table, -1)), -1)
    _count(refs, new, 1)
    # the page that the next token goes to, where it is partly filled: the
    # lowest of its rows keeps it if nobody else holds it, the others copy it
    row = torch.arange(R, device=table.device)
    part = n % bs != 0
    tail = torch.where(part, new[row, n // bs].long(), torch.full_like(n, blocks))
    rows_of = torch.zeros(blocks + 1, dtype=torch.long, device=table.device).index_add_(0, tail, torch.ones_like(tail))
    lowest = torch.full((blocks + 1,), R, dtype=torch.long, device=table.device).scatter_reduce_(0, tail, row, "amin")
    held_by = torch.cat([refs.long(), refs.new_zeros(1).long()])
    copy = part & ((row != lowest[tail]) | (held_by[tail] > rows_of[tail]))
    more = (n + grow + bs - 1) // bs - held
    need = copy.long() + more
    off = torch.cumsum(need, 0) - need
    free = torch.nonzero(refs == 0)[:, 0]
    served = (need == 0) | (off + need <= free.numel())
    take = torch.arange(int(need.max()), device=table.device)
    ids = torch.cat([free, free.new_zeros(1)])[(off[:, None] + take).clamp(max=free.numel())]
    mine = served[:, None] & (take < need[:, None])
    place = torch.where(copy[:, None] & (take == 0), (n // bs)[:, None], held[:, None] + take - copy.long()[:, None])
    copy = copy & served
    _count(refs, torch.where(copy, tail, torch.full_like(tail, -1)), -1)
    refs[ids[mine]] = 1
    new[row[:, None].expand_as(ids)[mine], place[mine]] = ids[mine].to(new.dtype)
    at = n[:, None] + torch.arange(grow, device=table.device)
    slots = torch.where(served[:, None], torch.gather(new.long(), 1, (at // bs).clamp(max=width - 1)) * bs + at % bs, torch.full_like(at, -1))
    copies = torch.where(copy[:, None], torch.stack([tail, ids[:, 0] if ids.shape[1] else tail], 1), torch.full((), -1, device=table.device)).to(torch.int32)
    taken = torch.where(served, need, torch.zeros_like(need)).sum()
    stats = torch.stack([free.numel() - taken, taken, (~served).sum(), copy.sum()]).to(torch.int32)
    return new, (n + torch.where(served, grow, 0)).to(torch.int32), slots, copies, stats


def _compact(x, table, length, refs):
    bs, blocks, width = x["case"]["bs"], x["blocks"], x["width"]
    live = refs > 0
    count = int(live.sum())
    holes = torch.nonzero(~live[:count])[:, 0]
    movers = (torch.nonzero(live[count:])[:, 0] + count).flip(0)
    remap = torch.where(live, torch.arange(blocks, device=table.device), torch.full((), -1, device=table.device))
    remap[movers] = holes
    in_use = (torch.arange(width, device=table.device) < ((length.long() + bs - 1) // bs)[:, None]) & (table >= 0)
    table = torch.where(in_use, remap[table.long().clamp(min=0)].to(table.dtype), table)
    refs[holes] = refs[movers]
    refs[movers] = 0
    copies = torch.full((blocks // 2, 2), -1, dtype=torch.int32, device=table.device)
    copies[:len(movers)] = torch.stack([movers, holes], 1).to(torch.int32)
    stats = torch.tensor([count, len(movers)], dtype=torch.int32, device=table.device)
    return table, copies, remap.to(torch.int32), stats


def _copy_blocks(pool, copies):
    src, dst = copies[copies[:, 0] >= 0].long().T
    pool[dst] = pool[src]


def run(x):
    case, dev = x["case"], "cuda"
    if case["path"] == "step" or case["path"] == "rows":
        if own and case["path"] == "step":
            x["fnpu"].mixed_attn_run(x["plan"], x["q"], x["k"], x["v"], x["out"], x["lse"])
        elif own:
            x["fnpu"].window_decode(x["desc"], case["window"], case["sinks"], x["ctx_dev"], x["bt_dev"], x["most"], x["q"], x["k"], x["v"],
                                    x["out"], x["lse"], x["workspace"])
        else:
            n, t = case["chunks"], case["chunks"] * case["chunk"]
            _attend(x, 0, n, 0, t, x["out"], x["lse"])
            _attend(x, n, n + case["decodes"], t, x["T"], x["out"], x["lse"])
        return {"out": x["out"], "lse": x["lse"]}
    if case["path"] == "beam":
        if not own:
            return _select(x)
        x["fnpu"].beam_select(x["logits"], x["scores"], x["out_scores"], x["out_parents"], x["out_tokens"], x["workspace"],
                              finished=x["finished"], end_token=END)
        return {"scores": x["out_scores"], "parents": x["out_parents"], "tokens": x["out_tokens"]}
    table, length, refs = _views(x, x["state"].clone())
    R, grow = x["R"], case["grow"]
    if case["path"] == "turn":
        if own:
            if case["window"]:
                x["fnpu"].pages_free(x["pages"], table, length, refs, window=case["window"], sinks=case["sinks"])
            new, new_length = torch.empty_like(table), torch.empty_like(length)
            slots = torch.empty((R, grow), dtype=torch.int64, device=dev)
            copies, stats = torch.empty((R, 2), dtype=torch.int32, device=dev), torch.empty(4, dtype=torch.int32, device=dev)
            x["fnpu"].pages_fork(x["pages"], table, length, refs, new, new_length, slots, copies, stats, x["workspace"], parents=x["parents"])
            x["fnpu"].kv_copy_blocks(x["desc"], copies, x["k"], x["v"])
        else:
            new, new_length, slots, copies, stats = _turn(x, table, length, refs)
            for pool in x["k"] + x["v"]:
                _copy_blocks(pool, copies)
        return {"table": new, "length": new_length, "refs": refs, "slots": slots, "copies": copies, "stats": stats, "k": x["k"], "v": x["v"]}
    if own:
        copies = torch.empty((x["blocks"] // 2, 2), dtype=torch.int32, device=dev)
        remap, stats = torch.empty(x["blocks"], dtype=torch.int32, device=dev), torch.empty(2, dtype=torch.int32, device=dev)
        x["fnpu"].pages_compact(x["pages"], table, length, refs, copies, remap, stats, x["workspace"])
        x["fnpu"].kv_copy_blocks(x["desc"], copies, x["k"], x["v"])
    else:
        table, copies, remap, stats = _compact(x, table, length, refs)
        for pool in x["k"] + x["v"]:
            _copy_blocks(pool, copies)
    return {"table": table, "refs": refs, "copies": copies, "remap": remap, "stats": stats, "k": x["k"], "v": x["v"]}


# -------------------------------------------------------------------- work

def work(case):
    if case["path"] == "beam":
        n = case["groups"] * case["beams"]
        # logits, scores and flags once; scores, parents and tokens of the chosen
        return {"bytes": n * (case["vocab"] * (2 if case["dtype"] == "bf16" else 4) + 5) + 12 * case["groups"] * case["select"],
                "flops": 3 * n * case["vocab"]}
    hq, hkv, d = HEADS[case["heads"]]
    bs = case["bs"]
    if case["path"] in ("step", "rows"):
        q, ctx, _ = (a.astype(np.int64) for a in _lengths(case))
        w, s, T, keys, pairs, pages = case["window"], case["sinks"], int(q.sum()), 0, 0, 0
        for n, c in zip(q.tolist(), ctx.tolist()):
            first = max(0, c - n - w + 1)                 # of the first query's window
            keys += c - first + min(s, first)
            p = np.arange(c - n, c)
            lo = np.maximum(0, p - w + 1)
            pairs += int((p + 1 - lo + np.minimum(s, lo)).sum())
            pages += int(_needed((c + bs - 1) // bs, first, s, bs).sum())
        # every visible row of K and V once, the table's entries, queries, outputs
        return {"bytes": keys * 4 * hkv * d + 4 * pages + T * hq * (4 * d + 4), "flops": 4 * hq * d * pairs}
    length, rows, count = _pages_of(case)
    R, width, block = len(rows), max(len(r) for r in rows), 4 * bs * hkv * d
    if case["path"] == "turn":
        # table and lengths read and written, parents, counts read, slots, copies; of R rows that each
        # follow a beam at random, and of their partly filled pages, a share of 1/e goes on alone
        moved = int(R * (1 - (1 - (1 - 1 / case["beams"]) ** case["beams"]))) if case["beams"] > 1 else 0
        return {"bytes": 8 * R * width + R * (12 + 8 * case["grow"] + 8) + 4 * count + moved * case["layers"] * 2 * block, "flops": 0}
    spare = case["spare"] * count + R * (1 + case["grow"])
    moved = int(count * spare / (count + spare))
    return {"bytes": 8 * R * width + 8 * count + moved * (16 + case["layers"] * 2 * block), "flops": 0}


# ------------------------------------------------------- the same in 64 bits

def exact(case, seed):
    if case["path"] in ("turn", "compact"):
        return None   # whole numbers and copies of rows: nothing is computed that could be nearer
    x = _inputs(case, seed)
    if case["path"] == "beam":
        B, W, V, K = case["groups"], case["beams"], case["vocab"], case["select"]
        out = torch.full((B, K), -math.inf, dtype=torch.float64, device="cuda")
        for g in range(B):
            logp = torch.log_softmax(x["logits"][g].double(), -1) + x["scores"][g].double()[:, None]
            done = x["finished"][g] > 0
            all_ = torch.cat([logp[~done].reshape(-1), x["scores"][g].double()[done]])
            top = torch.topk(all_, min(K, all_.numel())).values
            out[g, :top.numel()] = top
        return {"scores": out, "parents": None, "tokens": None}
    hq, hkv, d = HEADS[case["heads"]]
    bs, w, s, G, at, outs, lses = case["bs"], case["window"], case["sinks"], hq // hkv, 0, [], []
    for i in range(len(x["ctx"])):
        n, c = int(x["q_len"][i]), int(x["ctx"][i])
        table = torch.from_numpy(x["bt"][i].astype(np.int64)).cuda()
        q = x["q"][at:at + n].double().view(n, hkv, G, d)
        at += n
        o, l = torch.empty((n, hkv, G, d), dtype=torch.float64, device="cuda"), torch.empty((n, hkv, G), dtype=torch.float64, device="cuda")
        for r in range(0, n, 256):
            p = torch.arange(c - n + r, c - n + min(n, r + 256), device="cuda")
            lo, hi = max(0, int(p[0]) - w + 1), int(p[-1]) + 1
            j = torch.cat([torch.arange(min(s, lo), device="cuda"), torch.arange(lo, hi, device="cuda")])
            kv = [x[name].view(-1, hkv, d)[table[j // bs] * bs + j % bs].double() for name in ("k", "v")]
            sc = torch.einsum("nhgd,chd->nhgc", q[r:r + 256], kv[0]) / math.sqrt(d)
            hidden = (j > p[:, None]) | ((j <= p[:, None] - w) & (j >= s))
            sc = sc.masked_fill(hidden[:, None, None, :], -math.inf)
            le = torch.logsumexp(sc, -1)
            l[r:r + 256] = le
            o[r:r + 256] = torch.einsum("nhgc,chd->nhgd", torch.exp(sc - le[..., None]), kv[1])
        outs.append(o.view(n, hq, d))
        lses.append(l.view(n, hq))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
