"""Attention weights and eviction over the 8-bit cache on the GPU against the
float64 reference.

Which tokens stay, where they move and every byte of the cache are exact.  Bounds of
the weights, fixed before the first run: a row's weight is 2^x of x = s scale
log2(e) - lse log2(e); with z the sum of |q||k| scale, x is off by z (2^-23 + 130 *
2^-24) for the logit (a sum of 128 exact products) and by 2^-22 (z + |lse|) for the
two products and their difference, the power by 2^-22, and a sum of m of them by
m 2^-24; the older weight is added with one rounding more.  Weights below 2^-126
may be zero.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_05742_amd as adapld
from test_gpu_kv4 import PAGES, bf16, f64, i32
from test_gpu_kv8 import arrays, fill, make_cache, rows_of

pytestmark = pytest.mark.gpu


# -------------------------------------------------------------------- weights

def filled(lens, page, Hkv, rng, max_pages=None, wide=1.0):
    """A cache of `lens` tokens in garbage, and each sequence's keys in float64."""
    cache, table = make_cache(lens, page, Hkv, rng, max_pages)
    n = max(max(lens), 1)
    k = bf16(rng.standard_normal((len(lens), n, Hkv, 128)) * wide)
    v = bf16(rng.standard_normal((len(lens), n, Hkv, 128)))
    adapld.kv8_append(cache, k.cuda(), v.cuda(), i32([0] * len(lens)), i32(lens))
    kc, ks, _, _ = arrays(cache)
    return cache, table, [oracle.kv8_rows(kc, ks, table[b], page, max(L, 0)) for b, L in enumerate(lens)]


def softmax_lse(q, keys, old, n, rows, T, G):
    """lse [B, Hq, T] of the new rows (0 for rows that are none), in float32."""
    B, _, Hq, D = q.shape
    lse = np.zeros((B, Hq, T), np.float32)
    for b in range(B):
        for i in range(n[b]):
            u = i if rows is None else rows[b][i]
            if not 0 <= u < T:
                continue
            for h in range(Hq):
                z = keys[b][h // G, :old[b] + i + 1] @ q[b, u, h] / math.sqrt(D)
                lse[b, h, u] = z.max() + math.log(np.exp(z - z.max()).sum())
    return lse


def check_weights(old, new, Hq, Hkv, T, page, rows=None, N=None, L_max=None, seed=0, wide=1.0, **kw):
    rng = np.random.default_rng(seed + T)
    B, G = len(old), Hq // Hkv
    L_max = max(new) if L_max is None else L_max
    cache, _, keys = filled(new, page, Hkv, rng, -(-max(L_max, 1) // page) + 1, wide)
    q = f64(bf16(rng.standard_normal((B, T, Hq, 128))))
    bound = T if rows is None else len(rows[0])
    m = [min(max(b - a, 0), bound if N is None else N) for a, b in zip(old, new)]
    lse = softmax_lse(q, keys, old, m, rows, T, G)
    if T > 2:
        lse[0, 0, T - 1] = -math.inf
    stride = L_max + 5
    w = rng.random((B, Hkv, stride)).astype(np.float32)
    p = rng.integers(-9, 99, (B, Hkv, stride)).astype(np.int32)
    first = rng.integers(0, 1000, B).tolist()
    want, wp, reach = oracle.kv8_attn_weights(q, lse, keys, old, new, first, w, p, rows, N)
    for in_place in (False, True):
        tw, tp = torch.from_numpy(w).cuda(), torch.from_numpy(p).cuda()
        out = tw if in_place else torch.full_like(tw, 7.5)
        got, gp = adapld.kv8_attn_weights(cache, bf16(q).cuda(), torch.from_numpy(lse).cuda(), i32(old), i32(new), i32(first), tw,
                                          tp, rows=None if rows is None else i32(rows), N=N, L_max=L_max, weights_out=out, **kw)
        assert got is out and gp is tp and np.array_equal(tp.cpu().numpy(), wp)
        got = f64(got)
        for b in range(B):
            end = old[b] + m[b]
            for g in range(Hkv):
                z = reach[b, g]
                top = np.abs(lse[b, g * G:(g + 1) * G][np.isfinite(lse[b, g * G:(g + 1) * G])]).max(initial=0)
                rel = z * (2.0 ** -23 + 130 * 2.0 ** -24) + 2.0 ** -22 * (z + top) + 2.0 ** -22 + (m[b] * G + 1) * 2.0 ** -24
                before = np.where(np.arange(end) < old[b], w[b, g, :end].astype(np.float64), 0.0)
                tol = rel * (want[b, g, :end] - before) + 2.0 ** -23 * want[b, g, :end] + m[b] * G * 2.0 ** -126
                assert (np.abs(got[b, g, :end] - want[b, g, :end]) <= tol).all(), (b, g)
            rest = w[b, :, end:] if in_place else 7.5
            assert (got[b, :, end:] == rest).all()
    return cache


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("T, Hq, Hkv", [(1, 4, 1), (1, 3, 3), (5, 8, 2), (9, 7, 1), (40, 4, 2)])
def test_weights(page, T, Hq, Hkv):
    old = [0, 31, 32, 127, 300 - T]
    check_weights(old, [o + max(1, T - b) for b, o in enumerate(old)], Hq, Hkv, T, page)


def test_weights_of_accepted_rows():
    """Rows picked from a tree, one twice, some outside; fewer than N; none at all;
    lengths that do not grow; a bound below them."""
    rows = [[3, 7, 19], [0, 0, 19], [20, 5, -1], [1, 2, 3], [4, 5, 6]]
    check_weights([100, 64, 10, 50, 50], [103, 66, 13, 50, 40], 8, 2, 20, 16, rows=rows)
    check_weights([100, 64, 10, 50, 50], [103, 66, 13, 51, 58], 8, 2, 20, 32, rows=rows, N=3, L_max=200)
    check_weights([90, 30], [99, 40], 4, 4, 12, 16, N=7)


@pytest.mark.parametrize("T, Hq, Hkv, L", [(256, 8, 1, 700), (100, 16, 2, 513), (256, 2, 2, 256)])
def test_weights_of_many_rows(T, Hq, Hkv, L):
    check_weights([L - T], [L], Hq, Hkv, T, 64)


@pytest.mark.parametrize("T, Hq, B", [(80, 8, 3), (7, 80, 3), (256, 8, 2)])
def test_weights_of_some_rows_over_long_contexts(T, Hq, B):
    """Rows that stay in LDS while several blocks of keys pass."""
    new = [9001, 8700, 4100][:B]
    check_weights([n - T for n in new[:-1]] + [new[-1] - 1], new, Hq, 8, T, 64)


def test_weights_of_many_accepted_rows():
    """Queries in any order, some twice, some that are none; fewer rows than the bound."""
    rng = np.random.default_rng(4)
    rows = rng.integers(-1, 32, (3, 24)).tolist()
    rows[0][3], rows[1][:] = 2 ** 31 - 1, [5] * 24
    check_weights([400, 90, 0], [424, 100, 7], 16, 4, 31, 32, rows=rows)


def test_weights_with_large_logits():
    check_weights([400, 20], [403, 23], 4, 1, 3, 16, wide=8.0)


@pytest.mark.parametrize("T, Hq, Hkv", [(5, 4, 2), (22, 4, 1), (20, 8, 1), (70, 4, 2)])
def test_weights_ignore_what_is_no_row(T, Hq, Hkv):
    """NaN in the queries and log-sum-exps that no row picks, in keys behind the length
    and in weights behind the old one changes nothing."""
    rng = np.random.default_rng(T)
    new, old = [200, 90], [200 - (T - 2), 90]
    cache, _, _ = filled(new, 16, Hkv, rng)
    rows = i32([[T - 1 - i for i in range(T - 2)], [0] * (T - 2)])
    q = bf16(rng.standard_normal((2, T, Hq, 128))).cuda()
    lse = torch.full((2, Hq, T), 6.0, device="cuda")
    w, p = torch.rand((2, Hkv, 224), device="cuda"), torch.zeros((2, Hkv, 224), dtype=torch.int32, device="cuda")
    call = lambda: adapld.kv8_attn_weights(cache, q, lse, i32(old), i32(new), i32([0, 0]), w, p, rows=rows,  # noqa: E731
                                           weights_out=torch.zeros_like(w))[0]
    want = call()
    assert torch.isfinite(want).all() and torch.equal(want[1, :, :90], w[1, :, :90])
    q[0, :2], q[1] = math.nan, math.nan
    lse[0, :, :2], lse[1] = math.nan, math.nan
    w[0, :, old[0]:] = math.nan
    assert torch.equal(call(), want)


@pytest.mark.parametrize("T, Hq, Hkv", [(4, 4, 4), (5, 4, 2), (24, 4, 1), (20, 8, 1), (70, 4, 2), (256, 2, 2)])
def test_weights_ignore_rows_without_keys(T, Hq, Hkv):
    """Heads whose log-sum-exp is -inf, or no number, give nothing, whatever their queries
    hold; a sequence may have no others."""
    rng = np.random.default_rng(T)
    new, old = [300, 300], [300 - T, 300 - T]
    cache, _, _ = filled(new, 16, Hkv, rng)
    q = bf16(rng.standard_normal((2, T, Hq, 128))).cuda()
    lse = torch.full((2, Hq, T), 6.0, device="cuda")
    off = torch.from_numpy(rng.random((Hq, T)) < 0.4).cuda()
    lse[0][off] = -math.inf
    lse[1] = -math.inf
    w, p = torch.rand((2, Hkv, 304), device="cuda"), torch.zeros((2, Hkv, 304), dtype=torch.int32, device="cuda")
    call = lambda: adapld.kv8_attn_weights(cache, q, lse, i32(old), i32(new), i32([0, 0]), w, p,  # noqa: E731
                                           weights_out=torch.zeros_like(w))[0]
    want = call()
    assert torch.isfinite(want).all()
    assert torch.equal(want[1, :, :old[1]], w[1, :, :old[1]]) and (want[1, :, old[1]:] == 0).all()
    q[0][off.T] = math.nan
    q[1] = math.inf
    assert torch.equal(call(), want)
    lse[lse == -math.inf] = math.nan
    assert torch.equal(call(), want)


@pytest.mark.parametrize("T, Hq, Hkv, B, L", [
    (4, 4, 4, 2, 300), (8, 4, 1, 2, 300), (50, 4, 4, 2, 300),    # up to 16, 32 and 64 stacked rows
    (24, 4, 1, 2, 300),                                          # rows that stay in LDS
    (20, 8, 1, 2, 300), (256, 2, 2, 2, 300),                     # the ring: 128 keys a workgroup
    (70, 16, 4, 8, 1990)])                                       # and 256
def test_weights_without_rows_that_see_a_nan(T, Hq, Hkv, B, L):
    """A NaN among the keys matters to the rows that give and see it, and to no others: it
    may lie in a kv head none of whose rows gives anything (sequence 0), or be a new key
    that only rows which give nothing see (sequence 1)."""
    rng = np.random.default_rng(T)
    G, page, old = Hq // Hkv, 16, L - T
    cache, table, _ = filled([L] * B, page, Hkv, rng)
    q = bf16(rng.standard_normal((B, T, Hq, 128))).cuda()
    lse = torch.full((B, Hq, T), 6.0, device="cuda")
    lse[0, :G, ::2], lse[0, :G, 1::2] = -math.inf, math.nan
    lse[1, -G:, 1:] = math.nan
    w, p = torch.rand((B, Hkv, L), device="cuda"), torch.zeros((B, Hkv, L), dtype=torch.int32, device="cuda")
    call = lambda: adapld.kv8_attn_weights(cache, q, lse, i32([old] * B), i32([L] * B), i32([0] * B), w, p,  # noqa: E731
                                           weights_out=torch.zeros_like(w))[0]
    want = call()
    assert torch.isfinite(want).all() and torch.equal(want[0, 0, :old], w[0, 0, :old])
    assert (want[0, 0, old:] == 0).all() and (want[1, -1, old + 1:] == 0).all() and want[1, -1, old] > 0
    for b, g, j in ((0, 0, 5), (0, 0, L - 1), (1, Hkv - 1, old + 1), (1, Hkv - 1, L - 1)):
        cache.k_codes[int(table[b][j // page]), g, j % page, 77] = 0x7f
    assert torch.equal(call(), want)


def test_weights_long_and_clamped():
    """Longer than one workgroup takes, several sequences; lengths outside are clamped."""
    rng = np.random.default_rng(5)
    L, Hq, Hkv = 9001, 4, 2
    cache, _, keys = filled([L, 700], 64, Hkv, rng)
    q = bf16(rng.standard_normal((2, 1, Hq, 128))).cuda()
    out, lse = adapld.tree_verify_attn_kv8(q, cache, i32([L, 700]), i32([1, 1]), L_max=L)
    w = torch.zeros((2, Hkv, L), device="cuda")
    p = torch.zeros((2, Hkv, L), dtype=torch.int32, device="cuda")
    adapld.kv8_attn_weights(cache, q, lse, i32([L - 1, 699]), i32([L, 700]), i32([0, 0]), w, p, L_max=L)
    for b, n in enumerate((L, 700)):
        z = torch.matmul(q[b, 0].double().view(Hkv, 2, 128), torch.from_numpy(keys[b]).cuda().transpose(1, 2)) / math.sqrt(128)
        want = z.softmax(-1).sum(1)
        # the attention's lse is within 1e-5 of the exact one (test_gpu_kv4.py's bound here), its weights so much off
        assert ((w[b, :, :n].double() - want).abs() <= 3e-5 * want).all() and (w[b, :, n:] == 0).all()
        assert (w[b].double().sum(-1) - 2).abs().max() <= 1e-4
    old = w.clone()
    adapld.kv8_attn_weights(cache, q, lse, i32([L + 7, -3]), i32([L + 8, -1]), i32([0, 0]), w, p, L_max=L)
    assert torch.equal(w, old)


# ------------------------------------------------------------------- eviction

def tensors(cache):
    return cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales


def check_evict(lens, budget, recent, page, Hkv, weights=None, positions=None, next_position=None, L_max=None, seed=0, bad=()):
    rng = np.random.default_rng(seed + budget)
    B = len(lens)
    L_max = max(lens) if L_max is None else L_max
    cache, table = make_cache([max(n, 0) for n in lens], page, Hkv, rng, -(-max(L_max, *lens) // page))
    n = max(max(lens), 1)
    k, v = rows_of(rng, B, n, Hkv, 12)
    adapld.kv8_append(cache, k.cuda(), v.cuda(), i32([0] * B), i32(lens))
    for b, i, page_id in bad:
        table[b, i] = page_id
    cache.page_table.copy_(i32(table))
    stride = L_max + 3
    w = rng.random((B, Hkv, stride)).astype(np.float32) if weights is None else weights(rng, (B, Hkv, stride)).astype(np.float32)
    p = np.stack([[rng.permutation(2 * stride)[:stride] for _ in range(Hkv)] for _ in range(B)]).astype(np.int32)
    p = p if positions is None else positions(p)
    nxt = [2 * stride] * B if next_position is None else next_position
    want = arrays(cache)
    clamped = [min(max(x, 0), L_max) for x in lens]
    wo, po, lo = oracle.kv8_evict(w, p, clamped, nxt, budget, recent, table, page, want)
    first = [t.clone() for t in tensors(cache)]
    for mode in ("out", "again", "in place"):
        if mode == "in place":
            for t, f in zip(tensors(cache), first):
                t.copy_(f)
        tw, tp, tl = torch.from_numpy(w).cuda(), torch.from_numpy(p).cuda(), i32(lens)
        a = dict(weights_out=torch.full_like(tw, 7.5), positions_out=torch.full_like(tp, 77), lens_out=torch.full_like(tl, 9))
        if mode == "in place":
            a = dict(lens_out=tl)
        gw, gp, gl = adapld.kv8_evict(cache, tw, tp, tl, i32(nxt), budget, recent, L_max=L_max, **a)
        assert gl.tolist() == lo
        for got, x in zip(arrays(cache), want):
            assert np.array_equal(got, x), mode
        gw, gp = gw.cpu().numpy(), gp.cpu().numpy()
        for b in range(B):
            for g in range(Hkv):
                m = lo[b]
                assert np.array_equal(gw[b, g, :m], np.array(wo[b * Hkv + g], np.float32)) and gp[b, g, :m].tolist() == po[b * Hkv + g]
                if mode != "in place":
                    assert (gw[b, g, m:] == 7.5).all() and (gp[b, g, m:] == 77).all()
                else:
                    assert np.array_equal(gw[b, g, m:], w[b, g, m:]) and np.array_equal(gp[b, g, m:], p[b, g, m:])


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("budget, recent", [(16, 0), (48, 16), (160, 160), (400, 30)])
def test_evict(page, budget, recent):
    check_evict([417, 400, 161, 3, 0, 300], budget, recent, page, 2)


@pytest.mark.parametrize("ties", ["few values", "zeros", "all equal", "signs"])
def test_evict_ties(ties):
    """Equal weights: the lowest slots stay, over more slots than a workgroup has threads."""
    make = {"few values": lambda r, s: r.integers(0, 4, s) / 4, "zeros": lambda r, s: r.random(s) * (r.random(s) < 0.2),
            "all equal": lambda r, s: np.full(s, 0.5),
            "signs": lambda r, s: r.choice(np.array([-0.0, 0.0, -1.0, 1.0, 1e-40, -1e-40]), s)}[ties]
    check_evict([2600, 1100], 1040, 100, 64, 1, weights=make)
    check_evict([2600, 1041], 1040, 0, 16, 2, weights=make)
    check_evict([70, 33, 32], 32, 5, 16, 3, weights=make)


def test_evict_sizes_of_weights():
    """Weights of any size: the digits of the selection."""
    check_evict([3000], 992, 64, 32, 3, weights=lambda r, s: np.exp2(r.uniform(-140, 120, s)))
    check_evict([3000], 992, 64, 32, 3, weights=lambda r, s: 1 + r.integers(0, 3000, s) * 2.0 ** -23)
    check_evict([300, 200], 32, 0, 32, 3, weights=lambda r, s: -np.exp2(r.uniform(-140, 120, s)))


def test_evict_not_a_number():
    """Infinities are ranked like other numbers, NaN as the largest or the smallest by
    its sign."""
    cache, _ = make_cache([64], 16, 1, np.random.default_rng(1))
    adapld.kv8_append(cache, *(bf16(np.ones((1, 64, 1, 128))).cuda() for _ in range(2)), i32([0]), i32([64]))
    w = torch.ones((1, 1, 64))
    w[0, 0, [3, 5]] = torch.tensor([math.nan, -math.nan])
    w[0, 0, [7, 9]] = torch.tensor([-math.inf, math.inf])
    w[0, 0, 48:] = torch.tensor([2.0, math.nan, math.inf, -math.inf] + [0.5] * 12)
    p = torch.arange(64, dtype=torch.int32, device="cuda").view(1, 1, 64)
    _, po, lo = adapld.kv8_evict(cache, w.cuda(), p, i32([64]), i32([64]), 48, 0)
    want = list(range(48))
    want[5], want[7], want[47] = 48, 49, 50      # -NaN, -inf and the last of the ones go
    assert lo.tolist() == [48] and po[0, 0, :48].tolist() == want


def test_evict_protection():
    """More protected tokens than the budget, all, none, positions at the ends of 32 bits."""
    check_evict([500, 480], 64, 700, 16, 2)
    check_evict([500, 480], 64, 2 ** 31 - 1, 16, 2, next_position=[-(2 ** 31), 2 ** 31 - 1])
    check_evict([500], 64, 0, 16, 2, next_position=[-5])
    ends = lambda p: np.where(p % 3 == 0, -(2 ** 31), np.where(p % 3 == 1, 2 ** 31 - 1, 0)).astype(np.int32)  # noqa: E731
    check_evict([500], 256, 10, 16, 2, positions=ends, next_position=[2 ** 31 - 1])


def test_evict_bounds():
    """Lengths outside are clamped; a bound at or below the budget; nothing to do."""
    check_evict([300, -4, 90], 32, 8, 16, 2, L_max=100)
    check_evict([60, 64, 10], 64, 8, 16, 2)
    check_evict([60, 64, 70], 64, 8, 16, 2, L_max=64)
    check_evict([16], 16, 16, 16, 1)
    check_evict([17], 16, 0, 16, 1)


def test_evict_pages_outside_the_pool():
    check_evict([300, 300], 128, 8, 16, 2, bad=[(0, 1, -1), (0, 3, 1 << 30), (0, 12, -5), (0, 17, 999)])


@pytest.mark.parametrize("lens, budget", [([5000, 4200], 4096), ([9000], 8192), ([8192], 8160), ([20000, 17000], 16400),
                                          ([33000], 800), ([80, 127, 64], 64)])
def test_evict_lengths(lens, budget):
    """Slots held a few, several or many a thread, more than a workgroup holds; many
    and few moves."""
    check_evict(lens, budget, 20, 64, 1)
    check_evict(lens, budget, 20, 64, 1, weights=lambda r, s: r.integers(0, 3, s))


def test_evict_many():
    check_evict([64 + 5 * b for b in range(40)], 64, 7, 16, 4)


def test_evict_offsets_beyond_32_bits():
    """Rows that move between the ends of a pool of more than 4 GiB an array."""
    page, Hkv = 256, 8
    n_pages = (5 << 30) // (page * Hkv * 128)
    cache = adapld.Kv8Cache.allocate(n_pages, page, Hkv, 1, 3)
    cache.page_table.copy_(i32([[n_pages - 1, 1, n_pages - 2]]))
    rng = np.random.default_rng(3)
    k, v = (bf16(rng.standard_normal((1, 700, Hkv, 128))).cuda() for _ in range(2))
    adapld.kv8_append(cache, k, v, i32([0]), i32([700]))
    w = torch.zeros((1, Hkv, 768), device="cuda")
    w[..., 40:60] = -1.0                     # these go, and the newest take their slots
    w[..., 680:700] = 1.0
    p = torch.arange(768, dtype=torch.int32, device="cuda").expand(1, Hkv, 768).contiguous()
    read = lambda c, s, j: c[cache.page_table[0, j // page], :, j % page].view(torch.float8_e4m3fn).float() * (  # noqa: E731
        s[cache.page_table[0, j // page], :, j % page // 16].int() << 23).view(torch.float32)[:, None]
    before = [[read(c, s, 680 + i) for i in range(20)] for c, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales))]
    _, po, lo = adapld.kv8_evict(cache, w, p, i32([700]), i32([700]), 672, 0)
    assert lo.tolist() == [672] and po[0, 3, 40:60].tolist() == list(range(680, 700)) and po[0, 0, :40].tolist() == list(range(40))
    for (c, s), rows in zip(((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)), before):
        for i in range(20):
            # re-rounded to at most a few scales more: half a step of E4M3's subnormals
            assert (read(c, s, 40 + i) - rows[i]).abs().max() <= 2.0 ** -10 * 2.0 ** -5


# ------------------------------------------------------------- the loop, graphs

def test_decoding_loop_with_a_bounded_cache():
    """Iterations as a server runs them: rotated queries and keys, the tree verified,
    accepted, its kept nodes appended, their weights added, tokens evicted and pages
    given back; the cache's bytes, tables and positions follow the reference, and the
    attention is that of the kept tokens."""
    rng = np.random.default_rng(71)
    B, Hkv, Hq, W, S, page, budget, cap = 3, 2, 8, 3, 3, 16, 64, 128
    T, G = W * (S + 1), Hq // Hkv
    cache = adapld.Kv8Cache.allocate(B * cap // page, page, Hkv, B, cap // page)
    fill(cache, rng)
    freqs = adapld.rope_frequencies(128)
    w = torch.zeros((B, Hkv, cap), device="cuda")
    p = torch.zeros((B, Hkv, cap), dtype=torch.int32, device="cuda")
    lens, seen = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    parent = np.array([-1 if u % (S + 1) == 0 else u - 1 for u in range(T)])
    depth = np.arange(T) % (S + 1)
    sees = np.array([[v // (S + 1) == u // (S + 1) and v <= u for v in range(T)] for u in range(T)])
    words = np.array([sum(1 << v for v in range(T) if sees[u, v]) for u in range(T)], dtype=np.int64)
    mask = torch.from_numpy(np.tile(words[None, :, None], (B, 1, 1))).cuda()
    tile = lambda x: i32(np.tile(x[None], (B, 1)).tolist())  # noqa: E731
    qw, kw = bf16(1 + 0.1 * rng.standard_normal(128)).cuda(), bf16(1 + 0.1 * rng.standard_normal(128)).cuda()

    def project(n, offsets):
        x = bf16(rng.standard_normal((B, n, (Hq + 2 * Hkv), 128))).cuda()
        q, k = adapld.qk_norm_rope(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], freqs, seen, offsets=offsets, q_weight=qw, k_weight=kw)
        return q, k, x[:, :, Hq + Hkv:].contiguous()

    def grow(k, v, new, rows, q, lse):
        """Appends up to new, adds weights, evicts, maps the pages; every step checked."""
        nonlocal lens, seen
        N = k.shape[1] if rows is None else rows.shape[1]
        _, granted = adapld.page_map(cache, lens, new)
        assert granted.tolist() == [1] * B
        table = cache.page_table.cpu().numpy()
        want = arrays(cache)
        r = None if rows is None else rows.tolist()
        oracle.kv8_append(f64(k), f64(v), lens.tolist(), new.tolist(), table, page, want, r)
        adapld.kv8_append(cache, k, v, lens, new, rows=rows)
        assert all(np.array_equal(a, b) for a, b in zip(arrays(cache), want))
        if q is not None:
            keys = [oracle.kv8_rows(want[0], want[1], table[b], page, int(n)) for b, n in enumerate(new)]
            ww, wp, _ = oracle.kv8_attn_weights(f64(q), lse.cpu().numpy(), keys, lens.tolist(), new.tolist(), seen.tolist(),
                                                f64(w), p.cpu().numpy(), r)
            adapld.kv8_attn_weights(cache, q, lse, lens, new, seen, w, p, rows=rows)
            assert np.allclose(f64(w), ww, rtol=1e-4, atol=1e-30) and np.array_equal(p.cpu().numpy(), wp)
        seen = seen + (new - lens)
        w0, p0 = w.cpu().numpy().copy(), p.cpu().numpy().copy()
        wo, po, lo = oracle.kv8_evict(w0, p0, new.tolist(), seen.tolist(), budget, 8, table, page, want)
        _, _, kept = adapld.kv8_evict(cache, w, p, new, seen, budget, 8)
        assert kept.tolist() == lo and all(np.array_equal(a, b) for a, b in zip(arrays(cache), want))
        for b in range(B):
            for g in range(Hkv):
                assert p[b, g, :lo[b]].tolist() == po[b * Hkv + g] and len(set(po[b * Hkv + g])) == lo[b]
        adapld.page_map(cache, new, kept)
        held = sum(-(-n // page) for n in lo)
        assert int(cache.free_count) == cache.n_pages - held
        lens = kept

    # prompts: the rows' own attention gives the first weights
    n0 = 40
    q, k, v = project(n0, None)
    prompt = i32([40, 1, 17])
    causal = torch.from_numpy(np.tile(np.array([(1 << (u + 1)) - 1 for u in range(n0)], np.int64)[None, :, None], (B, 1, 1))).cuda()
    _, lse = adapld.tree_verify_attn_kv8(q, cache, lens, prompt, k_tree=k, v_tree=v, tree_mask=causal)
    grow(k, v, prompt, None, q, lse)
    for it in range(12):
        q, k, v = project(1, None)          # the root token of the iteration
        root = adapld.tree_verify_attn_kv8(q, cache, lens, i32([1] * B), k_tree=k, v_tree=v,
                                           tree_mask=torch.ones((B, 1, 1), dtype=torch.int64, device="cuda"))
        grow(k, v, lens + 1, None, q, root[1])
        q, kt, vt = project(T, tile(depth))
        counts = i32([T, T - 3, 1])
        out, lse = adapld.tree_verify_attn_kv8(q, cache, lens, counts, k_tree=kt, v_tree=vt, tree_mask=mask)
        kc, ks, vc, vs = arrays(cache)
        table = cache.page_table.cpu().numpy()
        n = int(lens.max())
        dk, dv = np.zeros((B, Hkv, n, 128)), np.zeros((B, Hkv, n, 128))
        for b in range(B):
            L = int(lens[b])
            dk[b, :, :L], dv[b, :, :L] = oracle.kv8_rows(kc, ks, table[b], page, L), oracle.kv8_rows(vc, vs, table[b], page, L)
        o, l, spread, _ = oracle.kv4_verify(f64(q), dk, dv, lens.tolist(), counts.tolist(), f64(kt), f64(vt), np.tile(sees[None], (B, 1, 1)))
        for b, t in enumerate(counts.tolist()):
            assert (np.abs(f64(out[b, :t]) - o[b, :t]) <= 2.0 ** -8 * np.abs(o[b, :t]) + (2.0 ** -8 + 2.0 ** -9) * spread[b, :t]).all()
            assert np.abs(f64(lse[b, :, :t]) - l[b, :, :t]).max() < 1e-4
        token, target = rng.integers(0, 2, (B, T)), rng.integers(0, 2, (B, T + 1))
        kept_n, nodes, _ = adapld.accept_greedy(i32(token.tolist()), tile(parent), tile(depth), counts, mask, i32(target.tolist()), lens)
        grow(kt, vt, lens + kept_n, nodes, q, lse)
    assert int(seen[0]) > budget and lens.tolist()[0] == budget
    adapld.page_map(cache, lens, torch.zeros_like(lens))
    assert sorted(cache.free_pages.tolist()) == list(range(cache.n_pages))


def test_graph_replays():
    """Append, attention, weights and eviction captured, replayed over new inputs with
    eager work between; a second graph with buffers of its own."""
    rng = np.random.default_rng(67)
    B, Hkv, Hq, T, page, L0, budget = 3, 2, 8, 6, 16, 200, 176

    def build(seed):
        r = np.random.default_rng(seed)
        new = [L0 + T, L0 - 20 + T, 30 + T]
        cache, _ = make_cache(new, page, Hkv, r)
        k0, v0 = (bf16(r.standard_normal((B, L0, Hkv, 128))).cuda() for _ in range(2))
        old = i32([n - T for n in new])
        adapld.kv8_append(cache, k0, v0, i32([0] * B), old)
        s = dict(cache=cache, old=old, new=i32(new), q=bf16(r.standard_normal((B, T, Hq, 128))).cuda(),
                 kt=bf16(r.standard_normal((B, T, Hkv, 128))).cuda(), vt=bf16(r.standard_normal((B, T, Hkv, 128))).cuda(),
                 w=torch.rand((B, Hkv, 256), device="cuda"), p=torch.arange(256, dtype=torch.int32, device="cuda").expand(B, Hkv, 256).contiguous(),
                 out=torch.zeros((B, T, Hq, 128), dtype=torch.bfloat16, device="cuda"), lse=torch.zeros((B, Hq, T), device="cuda"),
                 counts=i32([T] * B), lens_out=i32([0] * B), w1=torch.zeros((B, Hkv, 256), device="cuda"),
                 w2=torch.zeros((B, Hkv, 256), device="cuda"), p2=torch.zeros((B, Hkv, 256), dtype=torch.int32, device="cuda"))
        need = adapld.workspace_bytes(adapld.OP_TREE_VERIFY_ATTN_KV8, B, 256, 0, 0, T, Hq, Hkv, 128)
        s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        s["ws2"] = torch.empty(adapld.kv8_evict_workspace_bytes(B, Hkv, 208, budget), dtype=torch.uint8, device="cuda")
        s["start"] = [t.clone() for t in tensors(cache)]
        return s

    def step(s):
        c = s["cache"]
        adapld.kv8_append(c, s["kt"], s["vt"], s["old"], s["new"])
        adapld.tree_verify_attn_kv8(s["q"], c, s["new"], s["counts"], L_max=208, out=s["out"], lse=s["lse"], ws=s["ws"])
        adapld.kv8_attn_weights(c, s["q"], s["lse"], s["old"], s["new"], s["old"], s["w"], s["p"], L_max=208, weights_out=s["w1"])
        adapld.kv8_evict(c, s["w1"], s["p"], s["new"], s["new"], budget, 16, L_max=208, weights_out=s["w2"],
                         positions_out=s["p2"], lens_out=s["lens_out"], ws=s["ws2"])

    def result(s):
        return [x.clone() for x in (*tensors(s["cache"]), s["out"], s["lse"], s["w1"], s["w2"], s["p2"], s["lens_out"])]

    def reset(s):
        for t, x in zip(tensors(s["cache"]), s["start"]):
            t.copy_(x)
        for n in ("out", "lse", "w1", "w2", "p2", "lens_out"):
            s[n].zero_()

    states, graphs = [build(1), build(2)], []
    for s in states:
        step(s)
        torch.cuda.synchronize()
        reset(s)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            step(s)
        torch.cuda.current_stream().wait_stream(side)
        graphs.append(g)
    for rep in range(4):
        want = []
        for s in states:
            reset(s)
            s["q"].mul_(1 + rep % 2)
            s["kt"].mul_(1.25)
            s["w"].copy_(torch.rand_like(s["w"]))
            step(s)
            torch.cuda.synchronize()
            want.append(result(s))
            reset(s)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, ww in zip(states, want):
            for a, b in zip(result(s), ww):
                assert torch.equal(a, b), rep


def test_other_stream():
    rng = np.random.default_rng(61)
    cache, _, _ = filled([300, 200], 16, 2, rng)
    q = bf16(rng.standard_normal((2, 3, 8, 128))).cuda()
    lse = torch.full((2, 8, 3), 6.0, device="cuda")
    w, p = torch.rand((2, 2, 320), device="cuda"), torch.arange(320, dtype=torch.int32, device="cuda").expand(2, 2, 320).contiguous()
    start = [t.clone() for t in tensors(cache)]
    res = []
    for stream in (None, torch.cuda.Stream()):
        for t, x in zip(tensors(cache), start):
            t.copy_(x)
        torch.cuda.synchronize()
        w1, pp = torch.zeros_like(w), p.clone()
        w2, p2 = torch.zeros_like(w), torch.zeros_like(p)
        torch.cuda.synchronize()
        adapld.kv8_attn_weights(cache, q, lse, i32([297, 198]), i32([300, 200]), i32([5, 6]), w, pp, weights_out=w1, stream=stream)
        r = adapld.kv8_evict(cache, w1, pp, i32([300, 200]), i32([300, 200]), 112, 10, weights_out=w2, positions_out=p2, stream=stream)
        torch.cuda.synchronize()
        res.append([x.clone() for x in (w1, pp, *r, *tensors(cache))])
    for a, b in zip(*res):
        assert torch.equal(a, b)
