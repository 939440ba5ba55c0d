"""A paged cache with rotary positions, in bf16 or 8 bits, held in device memory.

``RotaryCache`` owns the pools and runs a layer's calls in the order in which a
model makes them: ``append`` (the queries and new keys of a fused projection's
output rotated, keys and values stored), then ``attend`` over the cache with a plan
that all layers of a step share. Torch provides the device memory and the
stream; all compute is in the library's kernels.
"""
from __future__ import annotations

from typing import Optional

from . import (KV_BF16, Plan, PlanOpts, RopeDesc, kv8_attn_plan, kv8_block_bytes, kv_read, make_desc, mixed_attn_plan,
               mixed_attn_replan, mixed_attn_run, rope_append)


class RotaryCache:
    """``rope`` and ``inv_freq`` (fp32 on the device, [rotary_dim / 2]) give the
    rotation; ``kv_format`` the cache: ``KV_BF16``, ``KV_INT8_BLOCK`` or
    ``KV_E4M3_BLOCK``."""

    def __init__(self, num_q_heads: int, num_kv_heads: int, head_dim: int, block_size: int, num_blocks: int, rope: RopeDesc,
                 inv_freq, kv_format: int = KV_BF16, device: str = "cuda"):
        import torch
        self.torch = torch
        self.heads = (num_q_heads, num_kv_heads, head_dim)
        self.desc = make_desc(num_q_heads, num_kv_heads, head_dim, head_dim, block_size, num_blocks)
        self.rope, self.inv_freq, self.kv_format = rope, inv_freq, kv_format
        if kv_format == KV_BF16:
            shape, dtype = (num_blocks, block_size, num_kv_heads, head_dim), torch.bfloat16
        else:
            shape, dtype = (num_blocks * kv8_block_bytes(self.desc, kv_format),), torch.uint8
        self.k, self.v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        self.plan_of = (bytes(self.desc), kv_format)  # what a plan over this cache was made for

    def _empty(self, stream, *outputs):
        """Outputs (shape, dtype) allocated on the stream that writes them: memory that
        the caching allocator gives out on another one may still be in use there."""
        if stream is not None and isinstance(stream, int):
            stream = self.torch.cuda.ExternalStream(stream, device=self.k.device)
        with self.torch.cuda.stream(stream):
            return [self.torch.empty(shape, dtype=dtype, device=self.k.device) for shape, dtype in outputs]

    def _own(self, plan: Plan) -> None:
        """Layers share a plan, caches of another shape or format do not: it reads by its
        own strides, and its block ids are of its own pool."""
        if (plan.shape, plan.kv_format) != self.plan_of:
            raise ValueError("the plan is of a cache of another shape or format")

    def append(self, qkv, positions, slot_mapping, stream=None):
        """Store a step's keys and values and return its rotated queries.
        qkv: bf16 [tokens, Hq + 2 Hkv, d]; positions int32 [axes, tokens] (one axis:
        [tokens] will do); slot_mapping int64 [tokens]."""
        hq, hkv, d = self.heads
        q, = self._empty(stream, ((qkv.shape[0], hq, d), qkv.dtype))
        rope_append(self.desc, self.rope, self.inv_freq, positions, qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], slot_mapping,
                    q, self.k, self.v, kv_format=self.kv_format, stream=stream)
        return q

    def plan(self, query_len, context_len, phase, block_table, plan: Optional[Plan] = None, opts: Optional[PlanOpts] = None,
             stream=None) -> Plan:
        """A plan of a step over this cache; ``plan``: one of an earlier step to
        rebuild (no allocation in the steady state)."""
        if plan is not None:
            self._own(plan)
            mixed_attn_replan(plan, query_len, context_len, phase, block_table, opts=opts, stream=stream)
            return plan
        if self.kv_format == KV_BF16:
            return mixed_attn_plan(self.desc, query_len, context_len, phase, block_table, opts=opts, stream=stream)
        return kv8_attn_plan(self.desc, self.kv_format, query_len, context_len, phase, block_table, opts=opts, stream=stream)

    def attend(self, plan: Plan, q, stream=None):
        """(out bf16 [tokens, Hq, d], lse fp32 [tokens, Hq]) of the planned step."""
        self._own(plan)
        if q.dtype is not self.torch.bfloat16:
            raise TypeError("queries are bf16")
        if q.shape != (plan.num_tokens, self.heads[0], self.heads[2]):  # (the outputs are of its size)
            raise ValueError(f"expected the {plan.num_tokens} planned queries, not {tuple(q.shape)}")
        out, lse = self._empty(stream, (q.shape, q.dtype), (q.shape[:2], self.torch.float32))
        mixed_attn_run(plan, q, self.k, self.v, out, lse, stream=stream)
        return out, lse

    def read(self, slots, stream=None):
        """The stored rows of ``slots``, as bf16 [n, Hkv, d] each."""
        _, hkv, d = self.heads
        k, v = self._empty(stream, *(2 * [((slots.shape[0], hkv, d), self.torch.bfloat16)]))
        kv_read(self.desc, slots, self.k, self.v, k, v, kv_format=self.kv_format, stream=stream)
        return k, v
