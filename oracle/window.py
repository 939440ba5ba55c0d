"""fp64 reference for attention with a sliding window and sinks.

TEST INFRASTRUCTURE, like the rest of ``oracle``: only ``tests/`` may import
it. It shares no code with the CUDA path.

A query at position p sees key j iff j <= p and (j > p - window or j < sinks).
"""
from __future__ import annotations

import math

import numpy as np


def visible(p, window, sinks):
    """The keys that a query at position p sees, ascending."""
    return [j for j in range(p + 1) if j > p - window or j < sinks]


def attend(q, k, v, table, first_position, block_size, window, sinks, scale=None):
    """Rows q [n, Hq, d] at positions first_position .. of one sequence over pools
    k, v [blocks, bs, Hkv, d]: (out [n, Hq, d], lse [n, Hq], weighted |v|
    [n, Hq, d], and each row's largest sum of |q_i k_i| scale over its keys [n, Hq])."""
    n, hq, d = q.shape
    hkv = k.shape[2]
    g = hq // hkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, mass, lse, reach = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.full((n, hq), -np.inf), np.zeros((n, hq))
    for i in range(n):
        at = np.array(visible(first_position + i, window, sinks))
        block, slot = np.asarray(table)[at // block_size], at % block_size
        for h in range(hkv):
            keys, values = k[block, slot, h].astype(np.float64), v[block, slot, h].astype(np.float64)
            rows = q[i, h * g:(h + 1) * g].astype(np.float64)
            s = rows @ keys.T * scale
            m = s.max(-1, keepdims=True)
            p = np.exp(s - m)
            z = p.sum(-1, keepdims=True)
            out[i, h * g:(h + 1) * g] = p / z @ values
            mass[i, h * g:(h + 1) * g] = p / z @ np.abs(values)
            lse[i, h * g:(h + 1) * g] = (m + np.log(z))[:, 0]
            reach[i, h * g:(h + 1) * g] = (np.abs(rows) @ np.abs(keys).T).max(-1) * scale
    return out, lse, mass, reach


def bounds(out, lse, mass, reach, d):
    """How far a computation may be off that rounds each weight and each output to
    bf16 once (half a step, 2^-8 of the value) and sums scores and weights in fp32.
    A score of d products is off by at most d 2^-23 of the sum of their magnitudes
    (each addition rounds or truncates), which moves the log-sum-exp by as much and a
    weight by twice that share; exp2, log2 and the sums of weights add 2^-20."""
    e = reach * d * 2.0 ** -23
    share = (2 * e + 2.0 ** -20)[..., None]
    to_out = mass * (2.0 ** -8 + share * (1 + 2.0 ** -8)) + np.abs(out) * 2.0 ** -8 + 1e-30
    to_lse = e + 2.0 ** -20 + np.abs(lse) * 2.0 ** -22
    return to_out * (1 + 2.0 ** -7), to_lse
