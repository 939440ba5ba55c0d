"""A beam search over a windowed, paged cache that stays on the device.

A small random transformer (no checkpoint: what it says means nothing) reads a prompt for
each request and continues it with several beams. Prompts are attended under a plan; then
every step is: the chosen beams' rows fork (``BeamCache.advance``), each layer appends
and attends, and ``beam_select`` chooses the next beams and tokens. Tokens, parents and pages never
go to the host; after two steps the loop is captured in a CUDA graph of two steps and
replayed.

  python examples/beam_search_loop.py [--requests N] [--beams N] [--tokens N] [--window N] ...
"""
import argparse
import os
import sys
import time

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

END = 2


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--heads", type=int, nargs=3, default=(28, 4, 128), metavar=("HQ", "HKV", "D"))
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=600, help="longest prompt")
    ap.add_argument("--tokens", type=int, default=64, help="tokens a beam, an even number")
    ap.add_argument("--window", type=int, default=256)
    ap.add_argument("--sinks", type=int, default=4)
    ap.add_argument("--block", type=int, default=16)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--eager", action="store_true", help="no CUDA graph")
    a = ap.parse_args(argv)

    import torch
    import paper_2606_04415_gb300 as fnpu
    from paper_2606_04415_gb300.beams import BeamCache

    hq, hkv, d = a.heads
    G, W, rows, hidden = a.requests, a.beams, a.requests * a.beams, hq * d
    gen = torch.Generator(device="cuda").manual_seed(a.seed)

    def weight(*shape):
        return (torch.randn(shape, device="cuda", generator=gen) * shape[-1] ** -0.5).to(torch.bfloat16)

    embed = weight(a.vocab, hidden) * hidden ** 0.5
    layers = [(weight((hq + 2 * hkv) * d, hidden), weight(hidden, hidden)) for _ in range(a.layers)]
    lens = np.zeros((G, W), np.int64)                      # beam 0 reads the prompt, the others are idle until they fork from it
    lens[:, 0] = np.random.default_rng(a.seed).integers(a.prompt // 3 + 1, a.prompt + 1, G)
    most, live = a.prompt + a.tokens, min(a.prompt + a.tokens, a.window + a.sinks) // a.block + 4
    blocks = int(sum(-(-n // a.block) for n in lens[:, 0])) + rows * live
    cache = BeamCache(hq, hkv, d, a.block, blocks, a.layers, rows, most, a.window, a.sinks)

    def model(x, attend):
        for i, (qkv, o) in enumerate(layers):
            y = (torch.nn.functional.rms_norm(x, (hidden,)) @ qkv.T).view(len(x), hq + 2 * hkv, d)
            z, _ = attend(i, *(p.contiguous() for p in y.split([hq, hkv, hkv], 1)))
            x = x + z.view(len(x), hidden) @ o.T
        return torch.nn.functional.rms_norm(x, (hidden,)) @ embed.T * 0.3

    prompt = torch.randint(0, a.vocab, (int(lens.sum()),), device="cuda", generator=gen)
    plan, slots = cache.admit(lens.reshape(-1))
    x = embed[prompt]
    logits = torch.zeros((G, W, a.vocab), dtype=torch.bfloat16, device="cuda")
    logits[:, 0] = model(x, lambda i, q, k, v: cache.prefill(plan, slots, i, q, k, v))[torch.from_numpy(np.cumsum(lens[:, 0]) - 1).cuda()]
    scores = torch.full((G, W), -float("inf"), device="cuda")
    scores[:, 0] = 0
    finished = torch.zeros((G, W), dtype=torch.uint8, device="cuda")
    space = torch.empty(fnpu.beam_select_workspace(G, W, a.vocab, W), dtype=torch.uint8, device="cuda")
    chosen = [torch.empty((G, W), dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
    history = torch.zeros((2, a.tokens, G, W), dtype=torch.int32, device="cuda")  # parents and tokens of every step
    at, short = torch.zeros((), dtype=torch.long, device="cuda"), torch.zeros((), dtype=torch.int32, device="cuda")

    def step():
        fnpu.beam_select(logits, scores, *chosen, space, finished=finished, end_token=END)
        best, parents, tokens = chosen
        row = parents.view(-1)
        history.index_copy_(1, at[None], torch.stack([parents, tokens])[:, None])
        at.add_(1)
        scores.copy_(best)
        finished.copy_((finished.view(-1)[row.long().clamp(min=0)].view(G, W) > 0) | (tokens == END))
        cache.advance(row)
        short.add_(cache.stats[2])                         # rows without a block: their tokens are not stored
        logits.copy_(model(embed[tokens.view(-1).long().clamp(min=0)], cache.attend).view(G, W, a.vocab))

    for _ in range(2):
        step()
    if a.tokens > 2 and not a.eager:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
            step()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(a.tokens // 2 - 1):
        if a.eager:
            step()
            step()
        else:
            graph.replay()
    torch.cuda.synchronize()
    spent = time.perf_counter() - t0
    if fnpu.check() != fnpu.FNPU_OK or fnpu.plan_check(plan) != fnpu.FNPU_OK:
        raise RuntimeError("device error flag raised")
    # the beams' tokens, from the last step back
    parents, tokens = (x.cpu().numpy() for x in history)
    text, row = np.zeros((G, W, a.tokens), np.int32), np.arange(rows).reshape(G, W)
    for t in range(a.tokens - 1, -1, -1):
        text[:, :, t] = tokens[t].reshape(-1)[row]
        row = parents[t].reshape(-1)[row]
    free, unserved = cache.stats[0].item(), short.item()
    print("%d requests x %d beams, %d tokens: %.1f us a step of %d layers; %d of %d blocks free, %d times a row found none" % (
        G, W, a.tokens, spent / max(1, a.tokens - 2) * 1e6, a.layers, free, blocks, unserved))
    return {"text": text, "scores": scores.cpu().numpy(), "cache": cache, "unserved": unserved}


if __name__ == "__main__":
    main()
