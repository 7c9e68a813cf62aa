"""The 4-bit verify attention over values of any finite size.

Logits that rise along the context make the weights outgrow the reference they
are taken against; with values near the largest that the cache holds, the sums
of weights times values must stay finite all the same.

Bounds as in test_gpu_kv4.py: the output's rounding and the weights' (2^-8 each,
the latter of the weighted mean of |v|) and twice the weights' relative error.
That is z (2^-23 + 130 * 2^-24) for the logits (z at most 45 here: 3.6e-4), 2^-19
for the exponent's rounding (arguments below 64), 2^-22 for the exponential
and n 2^-28 for the sum (n below 2^12): 2^-10 covers it.  Logarithms carry the
same error once.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_05742_amd as adapld
from test_gpu_kv4 import Case, f64, i32

pytestmark = pytest.mark.gpu

DELTA = 2.0 ** -10
LEVELS = (0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # what E2M1 holds


def _rising(B, L, Hkv, T, G, v_size, tree, seed):
    """Sequences that share their pages.  Key j is level c_j of one sign vector,
    c_j = 0 for the first 256 keys and rising to 6; a query row is that sign
    vector times a height, so its logit of key j is the height's share c_j / 6.
    Returns the arguments and, per kv head, the values of K and V."""
    rng = np.random.default_rng(seed)
    page, D, Hq = 64, 128, Hkv * G
    n_pages = -(-L // page)
    cache = adapld.Kv4Cache.allocate(n_pages, page, Hkv, B, n_pages)
    cache.page_table.copy_(torch.arange(n_pages, dtype=torch.int32, device="cuda").expand(B, -1))
    sign = np.where(rng.random((Hkv, D)) < 0.5, -1.0, 1.0)
    level = np.zeros(L)
    level[256:] = np.array(LEVELS)[np.arange(L - 256) * len(LEVELS) // (L - 256)]
    k = level[:, None, None] * sign
    v = rng.choice(np.array([0.5, 1.0, 2.0, 3.0, 4.0, 6.0]), (L, Hkv, D)) * np.where(rng.random((L, Hkv, D)) < 0.5, -1, 1)
    v[..., ::32] = 6.0                       # one sign: their mean is the largest value itself
    v *= 2.0 ** v_size
    to = lambda x: torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda()  # noqa: E731
    slots = torch.arange(L, dtype=torch.int32, device="cuda")[None]
    adapld.kv4_append(cache, to(k[None]), to(v[None]), slots)
    kq, vq = (f64(x[0]) for x in adapld.kv4_gather(cache, slots))
    assert np.array_equal(kq, k) and np.array_equal(vq, v)          # on the grid
    # the height (log2 units) of each row: below and above what makes a step be done again
    height = rng.choice(np.array([-30.0, 3.0, 9.0, 11.5, 14.0, 20.0, 22.0, 40.0, 60.0]), (B, T, Hq, 1))
    q = height / (6 * 128 / math.sqrt(128) * math.log2(math.e)) * np.repeat(sign, G, 0)
    args = dict(q=to(q), cache=cache, lens=i32([L] * B), node_count=i32([T] * B), L_max=L)
    if tree:
        args["k_tree"] = to(rng.standard_normal((B, T, Hkv, D)) * 0.25)
        args["v_tree"] = to(rng.choice(np.array([-1.0, 0.5, 1.0]), (B, T, Hkv, D)) * 2.0 ** (v_size + 1))
        words = np.array([[sum(1 << (v % 64) for v in range(u + 1) if v // 64 == w) for w in range((T + 63) // 64)]
                          for u in range(T)], dtype=np.uint64)
        args["tree_mask"] = torch.from_numpy(np.tile(words.view(np.int64), (B, 1, 1))).cuda()
    return args, k, v


@pytest.mark.parametrize("v_size", (125, 108, 0, -60))
@pytest.mark.parametrize("T, G, Hkv, B, tree", [
    (1, 4, 4, 64, False), (4, 4, 4, 64, True),      # 16 rows
    (7, 4, 4, 64, True), (15, 4, 4, 64, True),      # 32 and 64 rows
    (30, 4, 4, 64, True), (64, 4, 4, 64, True),     # 128 and 256 rows
    (30, 4, 2, 1, True), (1, 4, 2, 2, False)])      # split contexts
def test_large_values_with_rising_logits(T, G, Hkv, B, tree, v_size):
    L = 3000
    args, k, v = _rising(B, L, Hkv, T, G, v_size, tree, T + B)
    out, lse = adapld.tree_verify_attn_kv4(**args)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    sees = np.tril(np.ones((1, T, T), bool)) if tree else None
    for b in sorted({0, B - 1}):
        g = b % Hkv
        heads = slice(g * G, (g + 1) * G)
        kt, vt = (f64(args[n])[b:b + 1, :, g:g + 1] if tree else None for n in ("k_tree", "v_tree"))
        o, l, spread, reach = oracle.kv4_verify(f64(args["q"])[b:b + 1, :, heads], k[None, None, :, g], v[None, None, :, g],
                                                [L], [T], kt, vt, sees)
        assert reach.max() <= 45
        got = f64(out[b, :, heads])
        tol = 2.0 ** -8 * np.abs(o[0]) + (2.0 ** -8 + 2 * DELTA) * spread[0]
        assert (np.abs(got - o[0]) <= tol).all(), (b, float((np.abs(got - o[0]) / tol).max()))
        assert (np.abs(f64(lse[b, heads]) - l[0]) <= 2.0 ** -22 * np.abs(l[0]) + DELTA).all(), b


def test_stored_infinities():
    """What append makes of infinities takes part like any other value."""
    L, Hkv, Hq, page = 600, 2, 8, 16
    cache = adapld.Kv4Cache.allocate(-(-L // page), page, Hkv, 1, -(-L // page))
    cache.page_table.copy_(torch.arange(cache.n_pages, dtype=torch.int32, device="cuda")[None])
    k = torch.zeros((1, L, Hkv, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.full((1, L, Hkv, 128), math.inf, dtype=torch.bfloat16, device="cuda")
    v[..., 1::2] = -math.inf
    adapld.kv4_append(cache, k, v, torch.arange(L, dtype=torch.int32, device="cuda")[None])
    for T in (1, 40):
        q = torch.randn((1, T, Hq, 128), device="cuda").to(torch.bfloat16)
        out, lse = adapld.tree_verify_attn_kv4(q, cache, i32([L]), i32([T]), L_max=L)
        # equal weights of an average of equal values: one rounding of a weight, one of the output
        assert ((out[..., 0::2].double() / (6 * 2.0 ** 125) - 1).abs() <= 2.0 ** -7).all()
        assert ((out[..., 1::2].double() / (-6 * 2.0 ** 125) - 1).abs() <= 2.0 ** -7).all()
        assert (lse.double() - math.log(L)).abs().max() <= 2.0 ** -20 * math.log(L)


@pytest.mark.parametrize("scale", (1e-42, 1e-30))
@pytest.mark.parametrize("T", (1, 7, 40))
def test_smallest_scales(T, scale):
    """Logits near 0, one of the scales subnormal: masked keys stay out."""
    c = Case([333, 41], 8, 2, T, [T, T], 16, 400, 137, tree="random")
    out, lse = c.run(scale=scale)
    c.check(out, lse, scale=scale)
