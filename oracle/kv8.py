"""fp64 reference for rotary positions and for the 8-bit cache with one
power-of-two scale per block of tokens and kv head.

TEST INFRASTRUCTURE, like the rest of ``oracle``: only ``tests/`` may import
it. It shares no code with the CUDA path.

Rotation of a pair (x1, x2) by the angle a = position * inv_freq:
(x1 cos a - x2 sin a, x2 cos a + x1 sin a). Pairs are (i, i + n/2) of the n
rotated columns, or neighbours.

Cache: a pool is bytes of num_blocks blocks; a block is codes [Hkv][bs][d], then
fp32 scales 2^e [Hkv], padded to 16 bytes. int8: value (code - 128) 2^e; e4m3:
value of the code times 2^e. e is the least integer with |x| <= largest 2^e for
all values of the block, in [-60, 60]; codes are nearest, ties to even. A run
(consecutive tokens at consecutive slots of one block) that does not begin at the
block's slot 0 keeps the larger exponent, and the rows before it are stored anew
from their stored values when it grows.
"""
from __future__ import annotations

import math

import numpy as np

from .fp8 import e4m3_value

INT8, E4M3 = 1, 2
LARGEST = {INT8: 127.0, E4M3: 448.0}
MIN_E, MAX_E = -60, 60
_VALUES = np.array([e4m3_value(c) for c in range(256)])
# finite non-negative e4m3 values ascending, and their codes
_POS = _VALUES[:127]


def rope(x, positions, inv_freq, pair_axis=None, offset=0, interleaved=False, inverse=False):
    """Rows [n, heads, d] in fp64, rotated; positions [axes, n]."""
    y = np.array(x, np.float64)
    f = np.asarray(inv_freq, np.float64)
    n = len(f)
    axis = np.zeros(n, int) if pair_axis is None else np.asarray(pair_axis, int)
    a = np.asarray(positions, np.float64)[axis].T * f
    a = -a if inverse else a
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    i = offset + (2 * np.arange(n) if interleaved else np.arange(n))
    j = i + (1 if interleaved else n)
    x1, x2 = y[:, :, i].copy(), y[:, :, j].copy()
    y[:, :, i], y[:, :, j] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


def block_bytes(hkv, bs, d):
    return hkv * bs * d + 16 * ((hkv + 3) // 4)


def views(pool, hkv, bs, d):
    """Codes [blocks, hkv, bs, d] and scales [blocks, hkv] of a pool's bytes (views)."""
    b = pool.reshape(-1, block_bytes(hkv, bs, d))
    codes = b[:, :hkv * bs * d].reshape(len(b), hkv, bs, d)
    scales = b[:, hkv * bs * d:hkv * bs * d + 4 * hkv].view(np.float32)
    assert np.shares_memory(codes, pool) and np.shares_memory(scales, pool)
    return codes, scales


def exponent(amax, fmt):
    """Least e with amax <= LARGEST 2^e, in range (by trial, exact)."""
    for e in range(MIN_E, MAX_E):
        if amax <= math.ldexp(LARGEST[fmt], e):
            return e
    return MAX_E


def encode(x, e, fmt):
    """Codes of fp64 values over 2^e."""
    v = np.ldexp(np.asarray(x, np.float64), -e)
    if fmt == INT8:
        return (np.rint(np.clip(v, -127, 127)) + 128).astype(np.uint8)
    a = np.minimum(np.abs(v), 448.0)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)        # least value >= a
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - a, a - _POS[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(np.signbit(v), code | 128, code).astype(np.uint8)


def decode(codes, fmt):
    return codes.astype(np.float64) - 128.0 if fmt == INT8 else _VALUES[codes]


def append(pool, rows, slots, hkv, bs, d, fmt):
    """Store fp64 rows [n, hkv, d] at ``slots`` (negative: skipped)."""
    codes, scales = views(pool, hkv, bs, d)
    t, n = 0, len(slots)
    while t < n:
        s = int(slots[t])
        if s < 0:
            t += 1
            continue
        blk, off, m = s // bs, s % bs, 1
        while t + m < n and off + m < bs and slots[t + m] == s + m:
            m += 1
        for h in range(hkv):
            new = rows[t:t + m, h]
            e = exponent(np.abs(new).max(), fmt)
            if off > 0:
                e0 = int(round(math.log2(scales[blk, h])))
                if e > e0:
                    old = np.ldexp(decode(codes[blk, h, :off], fmt), e0)
                    codes[blk, h, :off] = encode(old, e, fmt)
                e = max(e, e0)
            codes[blk, h, off:off + m] = encode(new, e, fmt)
            scales[blk, h] = math.ldexp(1.0, e)
        t += m


def read(pool, slots, hkv, bs, d, fmt):
    """Stored rows [n, hkv, d] in fp64 (zero for negative slots)."""
    codes, scales = views(pool, hkv, bs, d)
    out = np.zeros((len(slots), hkv, d))
    for i, s in enumerate(slots):
        if s >= 0:
            out[i] = decode(codes[s // bs, :, s % bs], fmt) * scales[s // bs][:, None]
    return out


def attention(q, query_len, context_len, block_table, k_pool, v_pool, hkv, bs, d, fmt, scale=None, tokens=None):
    """Causal attention of packed fp64 queries [T, Hq, d] over the stored
    values: (out [T, Hq, d], lse [T, Hq]); ``tokens``: of these rows only."""
    scale = d ** -0.5 if scale is None else scale
    T, hq, _ = q.shape
    G = hq // hkv
    out, lse = np.zeros((T, hq, d)), np.zeros((T, hq))
    at = 0
    for s, (n, c) in enumerate(zip(query_len, context_len)):
        n, c = int(n), int(c)
        mine = [i for i in range(n) if tokens is None or at + i in tokens]
        if mine:
            pos = np.arange(c)
            sl = np.asarray(block_table)[s, pos // bs].astype(np.int64) * bs + pos % bs
            k, v = read(k_pool, sl, hkv, bs, d, fmt), read(v_pool, sl, hkv, bs, d, fmt)
            for i in mine:
                see = c - n + i + 1
                for h in range(hq):
                    x = (k[:see, h // G] @ q[at + i, h]) * scale
                    m = x.max()
                    w = np.exp(x - m)
                    out[at + i, h] = (w @ v[:see, h // G]) / w.sum()
                    lse[at + i, h] = m + math.log(w.sum())
        at += n
    return out, lse


def attention_bound(q, query_len, context_len, block_table, k_pool, v_pool, hkv, bs, d, fmt, staged, scale=None, tokens=None):
    """As ``attention``, and how far a computation in fp32 with weights rounded once may be
    off: (out, lse, bound [T, Hq, d]). ``staged[s]``: sequence s attends over a bf16 copy of
    its blocks (weights in bf16), else over the codes (weights in f16).

    With p_j the softmax weights and u = 2^-9 (bf16) or 2^-11 (f16), weight j is off by at
    most u p_j. In f16 there is a least step too: weights are w_j = c p_j 2^e_j with e_j the
    exponent of the block's V scale and the largest w at least 1, so a code enters with
    an error of 2^-25 / c at most, 1 / c <= max_i p_i 2^e_i. Roundings of different
    weights are independent: the sum of n terms within a_j exceeds 7 sqrt(sum a_j^2)
    with probability 2 exp(-49 / 2) < 5e-11 (Hoeffding). Row sums may take the rounded
    weights or the exact ones, so a term is a weight's error times |v_j| + |out|. Scores are
    good to the 2e-5 max(1, |lse|) that the log-sum-exp is held to; errors e_j of them move
    the result by sum p_j e_j (v_j - out). The result is rounded to bf16, 2^-8 of it."""
    scale = d ** -0.5 if scale is None else scale
    T, hq, _ = q.shape
    G = hq // hkv
    out, lse, bound = np.zeros((T, hq, d)), np.zeros((T, hq)), np.full((T, hq, d), np.inf)
    at = 0
    for s, (n, c) in enumerate(zip(query_len, context_len)):
        n, c = int(n), int(c)
        mine = [i for i in range(n) if tokens is None or at + i in tokens]
        if mine:
            pos = np.arange(c)
            sl = np.asarray(block_table)[s, pos // bs].astype(np.int64) * bs + pos % bs
            k, v = read(k_pool, sl, hkv, bs, d, fmt), read(v_pool, sl, hkv, bs, d, fmt)
            unit = views(v_pool, hkv, bs, d)[1][sl // bs].astype(np.float64)  # 2^e of each key and head
            a, a2, code2 = np.abs(v), v * v, (v / unit[:, :, None]) ** 2
            for i in mine:
                see = c - n + i + 1
                for h in range(hq):
                    kv = h // G
                    x = (k[:see, kv] @ q[at + i, h]) * scale
                    m = x.max()
                    w = np.exp(x - m)
                    p = w / w.sum()
                    o = p @ v[:see, kv]
                    out[at + i, h], lse[at + i, h] = o, m + math.log(w.sum())
                    p2, size = p * p, np.abs(o)
                    terms = p2 @ a2[:see, kv] + 2 * size * (p2 @ a[:see, kv]) + size ** 2 * p2.sum()
                    var = terms * (2.0 ** -18 if staged[s] else 2.0 ** -22)
                    if not staged[s]:
                        var = var + (2.0 ** -25 * (p * unit[:see, kv]).max()) ** 2 * code2[:see, kv].sum(0)
                    bound[at + i, h] = (2.0 ** -8 * size + 7 * np.sqrt(var) +
                                        2e-5 * max(1.0, abs(lse[at + i, h])) * (p @ np.abs(v[:see, kv] - o)))
        at += n
    return out, lse, bound
