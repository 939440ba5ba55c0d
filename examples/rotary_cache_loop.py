"""A serving loop over a rotary cache in 8 bits: prompts in chunks, then tokens.

Sequences of unequal prompts join one by one. Each step plans the batch once (one
chunk of a prompt beside the tokens of the sequences that are through theirs), then
for every layer appends the projection's rows with their rotation and attends over
the cache. A second cache in bf16 takes the same rows, and the two outputs are
compared. Projections are random (the loop has no model): what it shows is the
order of the calls and what the 8-bit cache costs in accuracy and time.

  python examples/rotary_cache_loop.py [--format int8|e4m3] [--sequences N] [--tokens N] ...
"""
import argparse
import os
import sys
import time

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--format", choices=("int8", "e4m3"), default="int8")
    ap.add_argument("--heads", type=int, nargs=3, default=(28, 4, 128), metavar=("HQ", "HKV", "D"))
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=700, help="longest prompt")
    ap.add_argument("--chunk", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=32, help="tokens a sequence")
    ap.add_argument("--block", type=int, default=16)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)

    import torch
    import paper_2606_04415_gb300 as fnpu
    from paper_2606_04415_gb300.rotary import RotaryCache

    hq, hkv, d = a.heads
    rng = np.random.default_rng(a.seed)
    gen = torch.Generator(device="cuda").manual_seed(a.seed)
    prompts = rng.integers(a.prompt // 3 + 1, a.prompt + 1, a.sequences)
    need = -(-(prompts + a.tokens) // a.block)
    blocks = rng.permutation(int(need.sum())).astype(np.int32)
    table = np.zeros((a.sequences, int(need.max())), np.int32)
    for s, at in enumerate(np.cumsum(need) - need):
        table[s, :need[s]] = blocks[at:at + need[s]]

    rope = fnpu.make_rope(d)
    inv_freq = torch.from_numpy((1e4 ** (-np.arange(d // 2) * 2.0 / d)).astype(np.float32)).cuda()
    formats = (fnpu.KV_INT8_BLOCK if a.format == "int8" else fnpu.KV_E4M3_BLOCK, fnpu.KV_BF16)
    caches = [[RotaryCache(hq, hkv, d, a.block, len(blocks), rope, inv_freq, f) for _ in range(a.layers)] for f in formats]
    plans, spent, worst, steps = [None, None], [0.0, 0.0], 0.0, 0

    done = np.zeros(a.sequences, np.int64)          # tokens of each sequence in the cache
    while (done < prompts + a.tokens).any():
        filling = np.flatnonzero(done < prompts)
        live = np.flatnonzero((done >= prompts) & (done < prompts + a.tokens))
        seqs = np.concatenate([filling[:1], live]).astype(int)
        qlen = np.array([min(a.chunk, prompts[s] - done[s]) if done[s] < prompts[s] else 1 for s in seqs], np.int32)
        ctx = (done[seqs] + qlen).astype(np.int32)
        phase = (done[seqs] >= prompts[seqs]).astype(np.uint8)
        pos = np.concatenate([np.arange(c - n, c) for n, c in zip(qlen, ctx)])
        row = np.repeat(seqs, qlen)
        slots = torch.from_numpy(table[row, pos // a.block].astype(np.int64) * a.block + pos % a.block).cuda()
        positions = torch.from_numpy(pos.astype(np.int32)).cuda()
        outs = []
        qkv = [torch.randn((len(pos), hq + 2 * hkv, d), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(a.layers)]
        for i, layers in enumerate(caches):
            torch.cuda.synchronize()
            t = time.perf_counter()
            plans[i] = layers[0].plan(qlen, ctx, phase, table[seqs], plan=plans[i])
            outs.append([c.attend(plans[i], c.append(x, positions, slots)) for c, x in zip(layers, qkv)])
            torch.cuda.synchronize()
            spent[i] += time.perf_counter() - t
        for (o, _), (b, _) in zip(*outs):
            worst = max(worst, float((o.float() - b.float()).norm() / b.float().norm()))
        done[seqs] += qlen
        steps += 1
    if any(fnpu.plan_check(p) != fnpu.FNPU_OK for p in plans) or fnpu.check() != fnpu.FNPU_OK:
        raise RuntimeError("device error flag raised")
    size = [sum(c.k.numel() * c.k.element_size() * 2 for c in layers) for layers in caches]
    print("%d steps of %d layers: %s cache %.1f us a step, %.1f MB; bf16 cache %.1f us, %.1f MB; outputs differ by up to %.2g" % (
        steps, a.layers, a.format, spent[0] / steps * 1e6, size[0] / 1e6, spent[1] / steps * 1e6, size[1] / 1e6, worst))
    return worst


if __name__ == "__main__":
    main()
