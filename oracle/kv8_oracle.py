"""CPU reference of the paged 8-bit K/V cache and the operators around it, in
float64 and plain Python.

Rows are quantised by looking up the nearest E4M3 value in its table, blocks and
evicted tokens are taken one at a time; nothing here shares code with the HIP path.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 16
MIN_EXP, MAX_EXP = 10, 246
# magnitude of codes 0..126 (127 is NaN): 4 bits of exponent with bias 7, 3 of fraction
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def kv8_codes(x, e):
    """Codes of float64 x at exponent byte e: nearest, ties to the even code,
    magnitudes above the largest as the largest, NaN as 0x7f."""
    x = np.asarray(x, np.float64)
    y = np.abs(x) / 2.0 ** (e - 127.0)
    y = np.where(np.isnan(y), 0.0, np.minimum(y, E4M3[-1]))
    hi = np.minimum(np.searchsorted(E4M3, y), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3[hi] - y, y - E4M3[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    return np.where(np.isnan(x), 127, code | (np.signbit(x).astype(np.uint8) << 7)).astype(np.uint8)


def kv8_values(codes, e):
    """float64 values of codes at exponent byte(s) e (broadcast)."""
    c = np.asarray(codes)
    m = np.where((c & 127) == 127, np.nan, E4M3[np.minimum(c & 127, 126)])
    return np.where(c & 128, -m, m) * 2.0 ** (np.asarray(e, np.float64) - 127.0)


def kv8_exponent(x):
    """The least e in 10..246 of which 448 * 2^(e - 127) holds every finite |x|."""
    x = np.abs(np.asarray(x, np.float64))
    x = x[np.isfinite(x)]
    amax = x.max() if x.size else 0.0
    e = MIN_EXP
    while e < MAX_EXP and 448.0 * 2.0 ** (e - 127) < amax:
        e += 1
    return e


def kv8_append(k, v, lens_old, lens_new, table, page, cache, rows=None, N=None):
    """Stores rows of k, v (float64 [B, n_src, Hkv, D]) into `cache`, the arrays
    (k_codes, k_scales, v_codes, v_scales), in place."""
    B, n_src, Hkv, D = k.shape
    N = (n_src if rows is None else len(rows[0])) if N is None else N
    n_pages, cap = cache[0].shape[0], len(table[0]) * page
    for b in range(B):
        old = min(max(int(lens_old[b]), 0), cap)
        new = min(min(max(int(lens_new[b]), 0), cap), old + N)
        if new <= old:
            continue
        for start in range(old // BLOCK * BLOCK, new, BLOCK):
            p, off = int(table[b][start // page]), start % page
            if not 0 <= p < n_pages:
                continue
            fresh = range(max(start, old), min(start + BLOCK, new))
            src = [i - old if rows is None else int(rows[b][i - old]) for i in fresh]
            for x, codes, scales in ((k, cache[0], cache[1]), (v, cache[2], cache[3])):
                got = np.stack([x[b, r] if 0 <= r < n_src else np.zeros((Hkv, D)) for r in src])
                for g in range(Hkv):
                    e, before, kept = kv8_exponent(got[:, g]), int(scales[p, g, off // BLOCK]), max(old - start, 0)
                    if kept:
                        e = max(e, before)
                        if e != before:
                            codes[p, g, off:off + kept] = kv8_codes(kv8_values(codes[p, g, off:off + kept], before), e)
                    at = off + fresh[0] - start
                    codes[p, g, at:at + len(src)] = kv8_codes(got[:, g], e)
                    scales[p, g, off // BLOCK] = e
    return cache


def kv8_rows(codes, scales, table, page, L):
    """float64 [Hkv, L, D]: the values of positions 0..L-1 of a table row."""
    out = np.zeros((codes.shape[1], L, codes.shape[3]))
    for j in range(L):
        p, off = int(table[j // page]), j % page
        out[:, j] = kv8_values(codes[p, :, off], scales[p, :, off // BLOCK][:, None])
    return out


def qk_norm_rope(x, weight, freqs, positions, eps, interleaved):
    """x float64 [tokens, heads, D] of bf16 values, weight float64 [D] or None,
    freqs as integers (turns per position in units of 2^-64), positions as
    integers: the rotated rows in float64, and the largest magnitude that takes
    part in each value."""
    out = np.array(x, np.float64)
    if weight is not None:
        out = out / np.sqrt((out * out).mean(-1, keepdims=True) + eps) * weight
    h = len(freqs)
    size = np.abs(out)
    for i, f in enumerate(freqs):
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        a = np.array([2 * math.pi * (((int(p) * int(f)) % (1 << 64)) / 2.0 ** 64) for p in positions])[:, None]
        y1, y2 = out[..., lo].copy(), out[..., hi].copy()
        out[..., lo] = y1 * np.cos(a) - y2 * np.sin(a)
        out[..., hi] = y2 * np.cos(a) + y1 * np.sin(a)
        size[..., lo] = size[..., hi] = np.abs(y1) + np.abs(y2)
    return out, size


def kv8_attn_weights(q, lse, keys, lens_old, lens_new, first_position, weights, positions, rows=None, N=None, scale=None):
    """q float64 [B, T, Hq, D], lse [B, Hq, T], keys a list of float64 [Hkv, L, D]
    (the values of each sequence's slots); weights float64 and positions int
    [B, Hkv, stride]: (weights, positions, reach) after the rows, reach the largest
    sum |q||k| * scale of each kv head, which bounds the rounding of a computation
    in fewer bits."""
    B, T, Hq, D = q.shape
    Hkv = weights.shape[1]
    G = Hq // Hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    N = (T if rows is None else len(rows[0])) if N is None else N
    w, p, reach = np.array(weights, np.float64), np.array(positions), np.zeros((B, Hkv))
    for b in range(B):
        old = int(lens_old[b])
        n = min(max(int(lens_new[b]) - old, 0), N)
        w[b, :, old:old + n] = 0.0
        p[b, :, old:old + n] = int(first_position[b]) + np.arange(n)
        for i in range(n):
            u = i if rows is None else int(rows[b][i])
            if not 0 <= u < T:
                continue
            for h in range(Hq):
                if lse[b, h, u] == -math.inf:
                    continue
                k = keys[b][h // G, :old + i + 1]
                w[b, h // G, :old + i + 1] += np.exp(k @ q[b, u, h] * scale - lse[b, h, u])
                reach[b, h // G] = max(reach[b, h // G], (np.abs(k) @ np.abs(q[b, u, h])).max() * scale)
    return w, p, reach


def kv8_evict(weights, positions, lens, next_position, budget, recent, table, page, cache):
    """One kv head after another; `cache` (the arrays k_codes, k_scales, v_codes,
    v_scales) is changed in place.  Returns (weights, positions, lens) of the
    tokens that stay, a list for each sequence and kv head, and the lengths."""
    B, Hkv = weights.shape[:2]
    n_pages = cache[0].shape[0]
    wo, po, lo = [], [], [min(max(int(n), 0), budget) for n in lens]
    for b in range(B):
        L, since = max(int(lens[b]), 0), int(next_position[b]) - recent
        for g in range(Hkv):
            w, p = weights[b, g, :L], positions[b, g, :L]
            src = list(range(min(L, budget)))
            if L > budget:
                # -0 is smaller than 0
                rank = sorted(range(L), key=lambda j: (int(p[j]) < since, -float(w[j]),
                                                       bool(np.signbit(w[j])), j))
                kept = set(rank[:budget])
                free = [j for j in range(budget) if j not in kept]
                for to, j in zip(free, sorted(j for j in kept if j >= budget)):
                    src[to] = j
                at = lambda j: (int(table[b][j // page]), g, j % page)  # noqa: E731
                near = lambda a: (min(max(a[0], 0), n_pages - 1), a[1], a[2])  # noqa: E731
                for codes, scales in ((cache[0], cache[1]), (cache[2], cache[3])):
                    for start in sorted({j // BLOCK * BLOCK for j in free}):
                        if not 0 <= at(start)[0] < n_pages:
                            continue
                        places = [near(at(src[j])) for j in range(start, start + BLOCK)]
                        es = [int(scales[x, g, y // BLOCK]) for x, _, y in places]
                        e = max(es)
                        got = [codes[x] if f == e else kv8_codes(kv8_values(codes[x], f), e) for x, f in zip(places, es)]
                        for i, c in enumerate(got):
                            codes[at(start + i)] = c
                        scales[at(start)[0], g, at(start)[2] // BLOCK] = e
            wo.append([w[j] for j in src])
            po.append([int(p[j]) for j in src])
    return wo, po, lo
