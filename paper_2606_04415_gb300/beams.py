"""The paged caches of a beam search, kept on the device.

``BeamCache`` owns the pools of all layers and the state of their pages: a block
table, lengths and counts of holders that all layers share. A step is ``advance`` (rows
continue the beams that were chosen, pages behind the window go, partly filled pages
that several rows would write to are copied), then ``attend`` a layer. Nothing
of it needs the host, so the steps can be captured in a CUDA graph -- two at a
time, as tables alternate between two buffers. All calls go to torch's current stream.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np

from . import (Plan, kv_append, kv_copy_blocks, make_desc, make_pages, mixed_attn_run, pages_compact, pages_fork, pages_free,
               pages_workspace, window_attn_plan, window_decode, window_decode_workspace)


class BeamCache:
    """``rows`` sequences over ``layers`` bf16 caches, of prompts of up to ``max_length``
    tokens, and of as many in all as whole blocks of ``max_length`` hold (``room``); ``window``
    (None: every query sees all earlier keys) and ``sinks`` as in ``window_attn_plan``."""

    def __init__(self, num_q_heads: int, num_kv_heads: int, head_dim: int, block_size: int, num_blocks: int, layers: int, rows: int,
                 max_length: int, window: Optional[int] = None, sinks: int = 0, device: str = "cuda"):
        import torch
        self.torch = torch
        self.heads, self.block_size, self.rows, self.max_length = (num_q_heads, num_kv_heads, head_dim), block_size, rows, max_length
        width = -(-max_length // block_size)
        self.room = width * block_size  # what pages_fork lets a row grow to
        self.window, self.sinks = window or max(1, self.room), sinks
        # A row that finds no block is attended at its old length, whose window begins one key
        # earlier than its next token's: the page of that key stays for one step more.
        self.freed_window = min(window, 2 ** 31 - 2) + 1 if window else 0
        self.desc = make_desc(num_q_heads, num_kv_heads, head_dim, head_dim, block_size, num_blocks)
        self.pages = make_pages(block_size, num_blocks)
        shape = (num_blocks, block_size, num_kv_heads, head_dim)
        self.k, self.v = ([torch.zeros(shape, dtype=torch.bfloat16, device=device) for _ in range(layers)] for _ in range(2))

        def state(*shape, fill=0):
            return torch.full(shape, fill, dtype=torch.int32, device=device)

        self.tables, self.lengths = [state(rows, width, fill=-1) for _ in range(2)], [state(rows) for _ in range(2)]
        self.refs, self.now = state(num_blocks), 0
        self.copies, self.stats, self.slots = state(rows, 2), state(4), torch.full((rows, 1), -1, dtype=torch.int64, device=device)
        self.moves, self.remap, self.moved = state(num_blocks // 2, 2), state(num_blocks), state(2)
        self.page_space = torch.empty(pages_workspace(self.pages, rows), dtype=torch.uint8, device=device)
        need = window_decode_workspace(self.desc, self.window, sinks, rows, self.room)
        self.decode_space = torch.empty(need, dtype=torch.uint8, device=device)

    @property
    def table(self):
        """Block table int32 [rows, width] of the step."""
        return self.tables[self.now]

    @property
    def length(self):
        """Tokens of each row, int32 [rows], the step's own among them."""
        return self.lengths[self.now]

    def admit(self, lengths: Sequence[int]):
        """Start over with prompts of ``lengths`` tokens (0: a row without one, as the
        idle beams of a request are). Returns (a plan of the prompts' attention, the slots of
        their tokens, int64 [tokens])."""
        n = np.asarray(lengths, np.int32)
        if n.shape != (self.rows,) or (n < 0).any() or (n > self.max_length).any():
            raise ValueError("a length of 0 .. max_length for every row")
        held = -(-n // self.block_size)
        if held.sum() > self.pages.num_blocks:
            raise ValueError("the prompts need %d blocks of %d" % (held.sum(), self.pages.num_blocks))
        table, first = np.full(tuple(self.table.shape), -1, np.int32), np.cumsum(held) - held
        for r in range(self.rows):
            table[r, :held[r]] = np.arange(first[r], first[r] + held[r])
        rows = np.flatnonzero(n)
        row, pos = np.repeat(rows, n[rows]), np.concatenate([np.arange(n[r]) for r in rows] + [np.zeros(0, np.int64)])
        slots = table[row, pos // self.block_size].astype(np.int64) * self.block_size + pos % self.block_size
        self.table.copy_(self.torch.from_numpy(table))
        self.length.copy_(self.torch.from_numpy(n))
        self.refs.zero_()
        self.refs[:int(held.sum())] = 1
        plan = window_attn_plan(self.desc, self.window, self.sinks, n[rows], n[rows], np.zeros(len(rows), np.uint8), table[rows])
        return plan, self.torch.from_numpy(slots).to(self.refs.device)

    def prefill(self, plan: Plan, slots, layer: int, q, k, v):
        """(out, lse) of a layer's prompts, whose keys and values are stored first."""
        kv_append(self.desc, k, v, slots, self.k[layer], self.v[layer])
        out, lse = self.torch.empty_like(q), self.torch.empty(q.shape[:2], dtype=self.torch.float32, device=q.device)
        mixed_attn_run(plan, q, self.k[layer], self.v[layer], out, lse)
        return out, lse

    def advance(self, parents) -> None:
        """Row r continues row parents[r] (int32 [rows] on the device; negative: an empty
        row), with room for its next token. ``stats`` then tells how many blocks are free,
        and how many rows found none or are at ``room`` (their slot is -1 and their length is as before)."""
        if self.freed_window:
            pages_free(self.pages, self.table, self.length, self.refs, window=self.freed_window, sinks=self.sinks)
        then = 1 - self.now
        pages_fork(self.pages, self.table, self.length, self.refs, self.tables[then], self.lengths[then], self.slots, self.copies,
                   self.stats, self.page_space, parents=parents)
        self.now = then
        kv_copy_blocks(self.desc, self.copies, self.k, self.v)

    def attend(self, layer: int, q, k, v):
        """(out bf16 [rows, Hq, d], lse fp32 [rows, Hq]) of the rows' next tokens, whose
        keys and values (bf16 [rows, Hkv, d]) are stored first. An empty row's are 0 and -inf."""
        kv_append(self.desc, k, v, self.slots.view(-1), self.k[layer], self.v[layer])
        out, lse = self.torch.empty_like(q), self.torch.empty(q.shape[:2], dtype=self.torch.float32, device=q.device)
        window_decode(self.desc, self.window, self.sinks, self.length, self.table, self.room, q, self.k[layer], self.v[layer], out,
                      lse, self.decode_space)
        return out, lse

    def end(self, rows) -> None:
        """Rows whose flag is set (uint8 [rows]) give up their pages and are empty then."""
        pages_free(self.pages, self.table, self.length, self.refs, ends=rows)

    def compact(self) -> None:
        """All live pages to the lowest ids; ``moved``: live blocks, blocks that moved. After a
        step's last layer: its ``slots`` and ``copies`` speak of the old places."""
        pages_compact(self.pages, self.table, self.length, self.refs, self.moves, self.remap, self.moved, self.page_space)
        kv_copy_blocks(self.desc, self.moves, self.k, self.v)
