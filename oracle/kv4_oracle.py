"""CPU reference of the paged 4-bit K/V cache, in float64 and plain Python.

Rows are quantised by trying every E2M1 code, pages move one at a time, and
attention is a softmax per row; nothing here shares code with the HIP path.
"""
from __future__ import annotations

import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def kv4_quantise(x):
    """x float64 [..., D] of bf16 values -> (codes 0..15 uint8 [..., D], scale
    bytes uint8 [..., D / 32]).  X = 2^(e - 127) is the smallest power of two
    with max|x| < 7 X, e in 1..252; codes are nearest, ties to the even code."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    amax = np.abs(g).max(-1)
    e = np.ones(amax.shape, np.int64)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):   # the largest e whose predecessor does not hold amax
        up = np.minimum(e + step, 252)
        e = np.where(amax >= 7.0 * np.exp2(up - 1.0 - 127), up, e)
    with np.errstate(over="ignore"):
        y = np.abs(g) / np.exp2(e - 127.0)[..., None]
    code = np.zeros(g.shape, np.uint8)
    best = np.abs(y - E2M1[0])
    for c in range(1, 8):
        d = np.abs(y - E2M1[c])
        win = (d < best) | ((d == best) & (c % 2 == 0))
        win |= np.isinf(y) & (c == 7)
        code = np.where(win, c, code).astype(np.uint8)
        best = np.where(win, d, best)
    code |= (np.signbit(g).astype(np.uint8) << 3)
    return code.reshape(x.shape), e.astype(np.uint8)


def kv4_pack(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def kv4_values(packed, scales):
    """Codes uint8 [..., D / 2] and scale bytes [..., D / 32] -> float64 [..., D]."""
    code = np.stack((packed & 15, packed >> 4), -1).reshape(*packed.shape[:-1], -1)
    v = np.where(code & 8, -E2M1[code & 7], E2M1[code & 7])
    return v * np.repeat(np.exp2(scales.astype(np.float64) - 127.0), GROUP, -1)


def kv4_page_map(lens_old, lens_new, page_size, page_table, free_pages, free_count, N):
    """One sequence after another; returns (page_table, free_pages, free_count,
    slot_map, granted) as new lists."""
    table = [list(map(int, r)) for r in page_table]
    stack = list(map(int, free_pages))
    max_pages = len(table[0])
    clamp = lambda v: min(max(int(v), 0), max_pages * page_size)  # noqa: E731
    pages = lambda v: -(-v // page_size)  # noqa: E731
    old, new = [clamp(v) for v in lens_old], [clamp(v) for v in lens_new]
    count = min(max(int(free_count), 0), len(stack))
    for b in range(len(old)):
        for i in range(pages(new[b]), pages(old[b])):
            if count < len(stack):
                stack[count] = table[b][i]
                count += 1
    asked, left = 0, count
    granted, slots = [], []
    for b in range(len(old)):
        need = max(pages(new[b]) - pages(old[b]), 0)
        asked += need
        ok = need == 0 or asked <= count
        granted.append(int(ok))
        row = [-1] * N
        if ok:
            for i in range(need):
                left -= 1
                table[b][pages(old[b]) + i] = stack[left]
            for i in range(min(N, max(new[b] - old[b], 0))):
                page = table[b][(old[b] + i) // page_size]
                if 0 <= page < len(stack):
                    row[i] = page * page_size + (old[b] + i) % page_size
        slots.append(row)
    return table, stack, left, slots, granted


def kv4_verify(q, k, v, lens, node_count, k_tree=None, v_tree=None, sees=None, scale=None):
    """Attention of every node in float64: q [B, T, Hq, D]; k, v [B, Hkv, L, D]
    the context's values; k_tree, v_tree [B, T, Hkv, D] and sees bool [B, T, T]
    or None.  Returns (out, lse, spread, reach): spread is the weighted mean of
    |value| and reach the largest sum |q||key| * scale of each row, which bound
    the rounding of a computation in fewer bits.  Rows past node_count are 0."""
    B, T_max, Hq, D = q.shape
    G = Hq // k.shape[1]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.zeros((B, Hq, T_max)), np.zeros((B, Hq, T_max))
    for b in range(B):
        L, T = int(lens[b]), int(node_count[b])
        for h in range(Hq):
            g = h // G
            for u in range(T):
                kk, vv = k[b, g, :L], v[b, g, :L]
                if sees is not None:
                    see = np.flatnonzero(sees[b, u, :T])
                    kk = np.concatenate((kk, k_tree[b, see, g]))
                    vv = np.concatenate((vv, v_tree[b, see, g]))
                if len(kk) == 0:
                    lse[b, h, u] = -math.inf
                    continue
                z = kk @ q[b, u, h] * scale
                m = z.max()
                w = np.exp(z - m)
                out[b, u, h] = w @ vv / w.sum()
                spread[b, u, h] = w @ np.abs(vv) / w.sum()
                lse[b, h, u] = m + math.log(w.sum())
                reach[b, h, u] = (np.abs(kk) @ np.abs(q[b, u, h])).max() * scale
    return out, lse, spread, reach
