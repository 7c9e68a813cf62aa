"""The 8-bit verify attention over values of any finite size.

Logits that rise along the context make the weights outgrow the reference they are
taken against; with values near the largest that the cache holds (448 * 2^119), the
sums of weights times values must stay finite all the same.  Bounds as in
test_gpu_kv4_range.py, whose kernels and roundings these are.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_05742_amd as adapld
from test_gpu_kv4 import f64, i32

pytestmark = pytest.mark.gpu

DELTA = 2.0 ** -10
LEVELS = (0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def to(x):
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("v_size", (127, 110, 0, -60))
@pytest.mark.parametrize("T, G, Hkv, B, tree", [
    (1, 4, 4, 64, False), (4, 4, 4, 64, True),      # 16 rows
    (7, 4, 4, 64, True), (15, 4, 4, 64, True),      # 32 and 64 rows
    (30, 4, 4, 64, True), (64, 4, 4, 64, True),     # 128 and 256 rows
    (30, 4, 2, 1, True), (1, 4, 2, 2, False)])      # split contexts
def test_large_values_with_rising_logits(T, G, Hkv, B, tree, v_size):
    """Sequences that share their pages.  Key j is level c_j of one sign vector, c_j = 0
    for the first 256 keys and rising to 6; a query row is that sign vector times a
    height, so its logit of key j is the height's share c_j / 6."""
    rng = np.random.default_rng(T + B)
    L, page, D, Hq = 3000, 64, 128, Hkv * G
    n_pages = -(-L // page)
    cache = adapld.Kv8Cache.allocate(n_pages, page, Hkv, 1, n_pages)
    cache.page_table.copy_(torch.arange(n_pages, dtype=torch.int32, device="cuda")[None])
    sign = np.where(rng.random((Hkv, D)) < 0.5, -1.0, 1.0)
    level = np.zeros(L)
    level[256:] = np.array(LEVELS)[np.arange(L - 256) * len(LEVELS) // (L - 256)]
    k = level[:, None, None] * sign
    v = rng.choice(np.array([0.5, 1.0, 1.5, 1.75]), (L, Hkv, D)) * np.where(rng.random((L, Hkv, D)) < 0.5, -1, 1)
    v[..., ::32] = 1.75                      # one sign: their mean is the largest value itself
    v *= 2.0 ** v_size
    adapld.kv8_append(cache, to(k[None]), to(v[None]), i32([0]), i32([L]))
    for codes, scales, x in ((cache.k_codes, cache.k_scales, k), (cache.v_codes, cache.v_scales, v)):
        rows = oracle.kv8_rows(codes.cpu().numpy(), scales.cpu().numpy(), np.arange(n_pages), page, L)
        assert np.array_equal(rows, x.transpose(1, 0, 2))          # on the grid
    cache.page_table = cache.page_table.expand(B, -1).contiguous()
    # the height (log2 units) of each row: below and above what makes a step be done again
    height = rng.choice(np.array([-30.0, 3.0, 9.0, 11.5, 14.0, 20.0, 22.0, 40.0, 60.0]), (B, T, Hq, 1))
    q = to(height / (6 * 128 / math.sqrt(128) * math.log2(math.e)) * np.repeat(sign, G, 0))
    args = dict(cache=cache, lens=i32([L] * B), node_count=i32([T] * B), L_max=L)
    sees = np.tril(np.ones((1, T, T), bool)) if tree else None
    if tree:
        words = np.array([[sum(1 << v for v in range(u + 1) if v // 64 == w) for w in range((T + 63) // 64)]
                          for u in range(T)], dtype=np.uint64)
        args |= dict(k_tree=to(rng.standard_normal((B, T, Hkv, D)) * 0.25),
                     v_tree=to(rng.choice(np.array([-1.0, 0.5, 1.0]), (B, T, Hkv, D)) * 2.0 ** v_size),
                     tree_mask=torch.from_numpy(np.tile(words.view(np.int64), (B, 1, 1))).cuda())
    out, lse = adapld.tree_verify_attn_kv8(q, **args)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    for b in sorted({0, B - 1}):
        g = b % Hkv
        heads = slice(g * G, (g + 1) * G)
        kt, vt = (f64(args[n])[b:b + 1, :, g:g + 1] if tree else None for n in ("k_tree", "v_tree"))
        o, l, spread, reach = oracle.kv4_verify(f64(q)[b:b + 1, :, heads], k[None, None, :, g], v[None, None, :, g],
                                                [L], [T], kt, vt, sees)
        assert reach.max() <= 45
        tol = 2.0 ** -8 * np.abs(o[0]) + (2.0 ** -8 + 2 * DELTA) * spread[0]
        assert (np.abs(f64(out[b, :, heads]) - o[0]) <= tol).all(), b
        assert (np.abs(f64(lse[b, heads]) - l[0]) <= 2.0 ** -22 * np.abs(l[0]) + DELTA).all(), b


def test_stored_infinities():
    """What append makes of infinities takes part like any other value."""
    L, Hkv, Hq, page = 600, 2, 8, 16
    cache = adapld.Kv8Cache.allocate(-(-L // page), page, Hkv, 1, -(-L // page))
    cache.page_table.copy_(torch.arange(cache.n_pages, dtype=torch.int32, device="cuda")[None])
    k = torch.zeros((1, L, Hkv, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.full((1, L, Hkv, 128), 1.75 * 2.0 ** 127, dtype=torch.bfloat16, device="cuda")
    v[:, 5::7] = math.inf
    v[..., 1::2] *= -1
    adapld.kv8_append(cache, k, v, i32([0]), i32([L]))
    for T in (1, 40):
        q = torch.randn((1, T, Hq, 128), device="cuda").to(torch.bfloat16)
        out, lse = adapld.tree_verify_attn_kv8(q, cache, i32([L]), i32([T]), L_max=L)
        # equal weights of an average of equal values: one rounding of a weight, one of the output
        assert ((out[..., 0::2].double() / (1.75 * 2.0 ** 127) - 1).abs() <= 2.0 ** -7).all()
        assert ((out[..., 1::2].double() / (-1.75 * 2.0 ** 127) - 1).abs() <= 2.0 ** -7).all()
        assert (lse.double() - math.log(L)).abs().max() <= 2.0 ** -20 * math.log(L)


@pytest.mark.parametrize("T", (1, 12, 50))
def test_a_nan_stays_in_its_head(T):
    rng = np.random.default_rng(T)
    L, Hkv, Hq, page = 300, 4, 8, 32
    cache = adapld.Kv8Cache.allocate(20, page, Hkv, 2, 10)
    cache.page_table.copy_(torch.arange(20, dtype=torch.int32, device="cuda").view(2, 10))
    k, v = (to(rng.standard_normal((2, L, Hkv, 128))) for _ in range(2))
    q = to(rng.standard_normal((2, T, Hq, 128)))
    run = lambda: adapld.tree_verify_attn_kv8(q, cache, i32([L, L]), i32([T, T]), L_max=L)  # noqa: E731
    adapld.kv8_append(cache, k, v, i32([0, 0]), i32([L, L]))
    out, lse = run()
    k[0, 77, 1, 5], v[0, 130, 1, 9] = math.nan, math.nan
    adapld.kv8_append(cache, k, v, i32([0, 0]), i32([L, L]))
    o2, l2 = run()
    others = [h for h in range(Hq) if h // 2 != 1]
    assert torch.equal(out[1], o2[1]) and torch.equal(lse[1], l2[1])
    assert torch.equal(out[0][:, others], o2[0][:, others]) and torch.equal(lse[0][others], l2[0][others])
