"""The paged 4-bit K/V cache on the GPU: pages, rows and the verify attention
against the float64 reference.

Bounds of the attention, fixed before the first run.  With A = sum p|v| / sum
p, one rounding of a weight to bf16 moves the output by at most 2^-8 A, the
final one by 2^-8 |out|.  The weights themselves are off by their logits'
error, z (2^-23 + 130 * 2^-24) for a sum of 128 exact products with z the sum
of |q||k| scale, and by the exponential (2^-22) and the fp32 sum of n weights (n /
16 * 2^-24 for sums of 16 lanes' runs): DELTA covers all of it for z <= 128 and n
<= 2^16 (2^-10), twice since numerator and denominator both carry it.  lse is
off by its own rounding and by that relative error of the sum, with the row's
own z and n.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_05742_amd as adapld

pytestmark = pytest.mark.gpu

DELTA = 2.0 ** -10
PAGES = (16, 32, 64, 128, 256)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------- pages

def _check_map(old, new, page, table, free, count, N, in_place=False):
    B, max_pages = len(old), len(table[0])
    cache = adapld.Kv4Cache.allocate(len(free), page, 1, B, max_pages)
    cache.page_table.copy_(i32(table))
    cache.free_pages.copy_(i32(free))
    cache.free_count.copy_(i32([count]))
    out = cache.free_count if in_place else torch.full((1,), -9, dtype=torch.int32, device="cuda")
    want = oracle.kv4_page_map(old, new, page, table, free, count, N)
    for _ in range(1 if in_place else 2):   # with another count buffer the call can be repeated
        slots = torch.full((B, N), -7, dtype=torch.int32, device="cuda")
        s, granted = adapld.page_map(cache, i32(old), i32(new), slot_map=slots, free_count_out=out)
        assert s is slots
        assert cache.page_table.tolist() == want[0]
        assert cache.free_pages.tolist() == want[1]
        assert out.tolist() == [want[2]]
        assert slots.tolist() == want[3]
        assert granted.tolist() == want[4]
    return cache


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("B, N, grow", [(1, 1, 1), (3, 5, 40), (64, 13, 13), (257, 40, 700), (1500, 3, 90)])
def test_page_map_random(page, B, N, grow):
    rng = np.random.default_rng(page * 1000 + B)
    max_pages = max(2, 900 // page + 1)
    top = max_pages * page
    old = rng.integers(0, max(top - grow, 1), B)
    new = np.where(rng.random(B) < 0.3, rng.integers(0, old + 1), np.minimum(old + rng.integers(0, grow + 1, B), top))
    held = -(-old // page)
    used = int(held.sum())
    n_pages = used + int(np.maximum(-(-new // page) - held, 0).sum()) + 3
    ids = rng.permutation(n_pages)
    table = np.full((B, max_pages), -1)
    at = 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    free = np.full(n_pages, -5)
    free[:n_pages - used] = ids[used:]
    _check_map(old.tolist(), new.tolist(), page, table.tolist(), free.tolist(), n_pages - used, N)
    # too few: only some of the free pages are on the stack
    _check_map(old.tolist(), new.tolist(), page, table.tolist(), free.tolist(), (n_pages - used) // 3, N, True)
    _check_map(old.tolist(), new.tolist(), page, table.tolist(), free.tolist(), 0, N, True)


def test_page_map_edges():
    # lengths outside the capacity are clamped, a count outside the pool too
    table = [[3, 1], [0, -1], [-1, -1]]
    _check_map([32, -5, 0], [900, 40, -2], 16, table, [2, 4, 5, -1, -1, -1], 3, 9)
    _check_map([32, 16, 0], [0, 0, 32], 16, table, [2, 4, 5, -1, -1, -1], 77, 4)
    _check_map([32, 16, 0], [0, 0, 32], 16, table, [2, 4, 5, -1, -1, -1], -3, 4)
    # nothing to do; no slots asked for; a table entry that is no page of the pool
    _check_map([5], [5], 16, [[0]], [1, -1], 1, 0)
    _check_map([5], [9], 16, [[7]], [1, -1], 1, 6)


def test_page_map_prompts():
    # many slots a sequence: the slot map is filled by a launch of its own
    rng = np.random.default_rng(9)
    old, new = [0, 100, 4000, 17, 0], [4096, 3000, 0, 2500, 1]
    table = np.full((5, 256), -1)
    ids = rng.permutation(1200)
    table[1, :7], table[2, :250], table[3, :2] = ids[:7], ids[7:257], ids[257:259]
    free = np.full(1200, -1)
    free[:941] = ids[259:]
    _check_map(old, new, 16, table.tolist(), free.tolist(), 941, 4097)


# ----------------------------------------------------------------------- rows

def _pool_bytes(cache):
    return [t.cpu().numpy().copy() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]


def _fill(cache, rng):
    for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        t.copy_(torch.from_numpy(rng.integers(0, 256, t.shape, dtype=np.uint8)))


def _check_append(k, v, slots, page, n_pages, rows=None):
    """Stored bytes are the reference's and no other byte moves; gather gives
    the values and leaves other rows."""
    rng = np.random.default_rng(11)
    B, n_src, Hkv, D = k.shape
    N = slots.shape[1]
    cache = adapld.Kv4Cache.allocate(n_pages, page, Hkv, 1, 1)
    _fill(cache, rng)
    want = _pool_bytes(cache)
    live = np.zeros((B, N), bool)
    for b in range(B):
        for i in range(N):
            s = int(slots[b, i])
            r = i if rows is None else int(rows[b, i])
            if 0 <= s < n_pages * page and 0 <= r < n_src:
                live[b, i] = True
                for x, c, e in ((k, 0, 1), (v, 2, 3)):
                    code, scale = oracle.kv4_quantise(f64(x[b, r]))
                    want[c][s // page, :, s % page], want[e][s // page, :, s % page] = oracle.kv4_pack(code), scale
    adapld.kv4_append(cache, k.cuda(), v.cuda(), i32(slots), rows=None if rows is None else i32(rows))
    for got, w in zip(_pool_bytes(cache), want):
        assert np.array_equal(got, w)
    ko = torch.full((B, N, Hkv, D), 77.0, dtype=torch.bfloat16, device="cuda")
    vo = ko.clone()
    adapld.kv4_gather(cache, i32(slots), k_out=ko, v_out=vo)
    for o, c, e in ((ko, 0, 1), (vo, 2, 3)):
        o = f64(o)
        for b in range(B):
            for i in range(N):
                s = int(slots[b, i])
                if live[b, i]:
                    assert np.array_equal(o[b, i], oracle.kv4_values(want[c][s // page, :, s % page], want[e][s // page, :, s % page]))
                elif not 0 <= s < n_pages * page:
                    assert (o[b, i] == 77.0).all()


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("B, N, Hkv", [(1, 1, 1), (2, 5, 3), (3, 37, 8), (1, 130, 2)])
def test_append_gather(page, B, N, Hkv):
    rng = np.random.default_rng(page + B + N)
    k = bf16(rng.standard_normal((B, N, Hkv, 128)) * np.exp2(rng.integers(-6, 6, (B, N, Hkv, 1))))
    v = bf16(rng.standard_normal((B, N, Hkv, 128)))
    n_pages = -(-B * N // page) + 2
    slots = rng.permutation(n_pages * page)[:B * N].reshape(B, N)
    slots[rng.random((B, N)) < 0.2] = -1
    _check_append(k, v, slots, page, n_pages)


def test_append_rows_and_padding():
    # accepted nodes: rows picked from the source; entries whose slot or row
    # is outside are skipped, whatever the other one holds
    rng = np.random.default_rng(21)
    k, v = bf16(rng.standard_normal((3, 9, 2, 128))), bf16(rng.standard_normal((3, 9, 2, 128)))
    slots = np.array([[5, 40, -1, 63], [0, 64, 1 << 30, -(1 << 31)], [17, 18, 19, 20]])
    rows = np.array([[8, 0, 3, 3], [4, 4, 4, 4], [9, -1, 7, 1 << 30]])
    _check_append(k, v, slots, 32, 2, rows)


def test_append_special_values():
    # zeros, signed zeros, ties, the bounds of the scale, subnormals, infinity
    rng = np.random.default_rng(23)
    x = np.zeros((1, 8, 1, 128), np.float32)
    x[0, 0, 0, 0] = -0.0
    x[0, 1, 0, :8] = [6.5, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    x[0, 1, 0, 32:38] = [7.0, -7.0, 0.5, 1.5, 6.0, 3.0]
    x[0, 2, 0] = rng.standard_normal(128) * 2.0 ** -130
    x[0, 3, 0, :4] = [3.3895314e38, -3.3895314e38, 1e38, 1.0]
    x[0, 4, 0, 5], x[0, 4, 0, 40] = math.inf, -math.inf
    x[0, 5, 0] = np.exp2(rng.integers(-40, 40, 128))
    x[0, 6, 0] = rng.standard_normal(128) * 2.0 ** -124
    x[0, 7, 0] = 2.0 ** -133
    _check_append(bf16(x), bf16(-x), np.arange(8)[None] + 3, 16, 1)


# ------------------------------------------------------------------ attention

class Case:
    """A cache filled through append, with a table of pages in random order and
    garbage (non-finite scales too) in every row that no sequence owns."""

    def __init__(self, lens, Hq, Hkv, T, counts, page, L_max, seed, tree=None, empty=0.2, wide=1.0):
        rng = self.rng = np.random.default_rng(seed)
        B = len(lens)
        self.lens, self.counts, self.T, self.Hq, self.Hkv = lens, counts, T, Hq, Hkv
        self.page, self.L_max = page, L_max
        D = 128
        max_pages = -(-L_max // page) + 1
        held = [-(-max(L, 0) // page) for L in lens]
        n_pages = sum(held) + 2
        ids = rng.permutation(n_pages)
        table = np.full((B, max_pages), -1)
        at = 0
        for b, n in enumerate(held):
            table[b, :n] = ids[at:at + n]
            at += n
        self.cache = adapld.Kv4Cache.allocate(n_pages, page, Hkv, B, max_pages)
        _fill(self.cache, rng)
        for t in (self.cache.k_scales, self.cache.v_scales):
            t[torch.rand(t.shape, device="cuda") < 0.3] = 255
        self.cache.page_table.copy_(i32(table))
        Lc = max(max(lens), 1)
        k = bf16(rng.standard_normal((B, Lc, Hkv, D)) * wide).cuda()
        v = bf16(rng.standard_normal((B, Lc, Hkv, D))).cuda()
        pos = np.arange(Lc)
        slots = np.full((B, Lc), -1)
        for b, L in enumerate(lens):
            slots[b, :max(L, 0)] = table[b, pos[:max(L, 0)] // page] * page + pos[:max(L, 0)] % page
        adapld.kv4_append(self.cache, k, v, i32(slots))
        kq, vq = adapld.kv4_gather(self.cache, i32(slots))
        self.kq, self.vq = kq.transpose(1, 2).contiguous(), vq.transpose(1, 2).contiguous()   # [B, Hkv, Lc, D]
        self.q = bf16(rng.standard_normal((B, T, Hq, D))).cuda()
        self.kt = self.vt = self.mask = self.sees = None
        if tree:
            self.kt, self.vt = (bf16(rng.standard_normal((B, T, Hkv, D))).cuda() for _ in range(2))
            if tree == "chain":
                sees = np.broadcast_to(np.tril(np.ones((T, T), bool)), (B, T, T)).copy()
            else:
                sees = rng.random((B, T, T)) < 0.4
                sees[:, np.arange(T), np.arange(T)] = True
                sees[rng.random((B, T)) < empty] = False     # rows that see the context alone
            self.sees = sees
            nw = (T + 63) // 64
            bits = np.zeros((B, T, nw * 64), np.uint64)
            bits[..., :T] = sees
            words = (bits.reshape(B, T, nw, 64) << np.arange(64, dtype=np.uint64)).sum(-1, dtype=np.uint64)
            self.mask = torch.from_numpy(words.view(np.int64)).cuda()

    def run(self, **kw):
        a = dict(k_tree=self.kt, v_tree=self.vt, tree_mask=self.mask, L_max=self.L_max) | kw
        return adapld.tree_verify_attn_kv4(self.q, self.cache, i32(self.lens), i32(self.counts), **a)

    def check(self, out, lse, lens=None, scale=None):
        L = [min(max(n, 0), self.L_max) for n in (lens or self.lens)]
        T = [min(max(n, 0), self.T) for n in self.counts]
        tree = (None, None, None) if self.kt is None else (f64(self.kt), f64(self.vt), self.sees)
        o, l, spread, reach = oracle.kv4_verify(f64(self.q), f64(self.kq), f64(self.vq), L, T, *tree, scale=scale)
        got, gl = f64(out), f64(lse)
        for b, t in enumerate(T):
            tol = 2.0 ** -8 * np.abs(o[b, :t]) + (2.0 ** -8 + 2 * DELTA) * spread[b, :t]
            bad = np.abs(got[b, :t] - o[b, :t]) > tol + 1e-30
            assert not bad.any(), (b, int(bad.sum()), float(np.abs(got[b, :t] - o[b, :t]).max()))
            n = L[b] + t
            want = l[b, :, :t]
            tol = 2.0 ** -22 * np.abs(want) + reach[b, :, :t] * (2.0 ** -23 + 130 * 2.0 ** -24) + 2.0 ** -22 + n * 2.0 ** -28
            empty = np.isinf(want)
            assert np.array_equal(gl[b, :, :t][empty], want[empty])
            assert (np.abs(gl[b, :, :t][~empty] - want[~empty]) <= tol[~empty]).all(), b


CASES = {
    # single tokens, no tree: every position of a length against page and tile
    "one_key": dict(lens=[1], Hq=4, Hkv=1, T=1, counts=[1], page=16, L_max=1),
    "decode_tails": dict(lens=[15, 16, 17, 63, 64, 65, 127, 129], Hq=8, Hkv=2, T=1, counts=[1] * 8, page=16, L_max=130),
    "decode_mha": dict(lens=[517, 33], Hq=6, Hkv=6, T=1, counts=[1, 1], page=32, L_max=517),
    "decode_g8_split": dict(lens=[2049, 1, 900], Hq=16, Hkv=2, T=1, counts=[1, 1, 1], page=128, L_max=2304),
    "decode_g5": dict(lens=[300], Hq=5, Hkv=1, T=3, counts=[3], page=256, L_max=300),
    # empty contexts, empty sequences, rows without any key
    "empty": dict(lens=[0, 5, 0, 70], Hq=4, Hkv=2, T=3, counts=[3, 0, 2, 3], page=16, L_max=70),
    "empty_tree": dict(lens=[0, 0, 130, 64], Hq=4, Hkv=2, T=9, counts=[9, 4, 0, 9], page=64, L_max=200, tree="random",
                       empty=0.5),
    # trees: chains, random masks, more rows than one workgroup, 256 nodes
    "chain16": dict(lens=[100, 99], Hq=8, Hkv=2, T=16, counts=[16, 16], page=32, L_max=128, tree="chain"),
    "tree_ragged": dict(lens=[640, 77, 321], Hq=14, Hkv=2, T=35, counts=[35, 1, 20], page=16, L_max=700, tree="random"),
    "tree_rows_256": dict(lens=[200], Hq=8, Hkv=1, T=33, counts=[33], page=64, L_max=256, tree="random"),
    "tree_136": dict(lens=[90, 191], Hq=10, Hkv=2, T=136, counts=[136, 70], page=128, L_max=192, tree="random"),
    "tree_256": dict(lens=[65], Hq=2, Hkv=1, T=256, counts=[256], page=16, L_max=80, tree="random"),
    "tree_split": dict(lens=[3000], Hq=4, Hkv=1, T=20, counts=[20], page=64, L_max=3000, tree="random"),
    "tree_batch": dict(lens=[33 + 41 * b for b in range(10)], Hq=8, Hkv=4, T=12, counts=[1 + b for b in range(10)],
                       page=32, L_max=512, tree="random"),
    # out-of-range lengths and counts are clamped
    "clamped": dict(lens=[50, -3, 64], Hq=4, Hkv=2, T=2, counts=[7, 2, -1], page=16, L_max=64, tree="chain"),
    # logits far apart: the running max moves often
    "wide": dict(lens=[700, 200], Hq=4, Hkv=1, T=5, counts=[5, 5], page=16, L_max=700, tree="random", wide=8.0),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_verify(name):
    c = Case(seed=len(name), **CASES[name])
    out, lse = c.run()
    c.check(out, lse)


@pytest.mark.parametrize("T, Hq, Hkv, tree", [(1, 8, 2, None), (7, 8, 2, "random"), (16, 8, 2, "chain"),
                                              (40, 8, 2, "random"), (70, 16, 2, "random")])
@pytest.mark.parametrize("page", PAGES)
def test_verify_pages(T, Hq, Hkv, tree, page):
    """Every page size gives the same bits, and so does a sequence alone."""
    lens, counts = [333, 64, 500], [T, max(T // 2, 1), T]
    c = Case(lens, Hq, Hkv, T, counts, page, 512, 5, tree=tree)
    out, lse = c.run()
    if page == 16:
        c.check(out, lse)
    d = Case(lens, Hq, Hkv, T, counts, 16, 512, 5, tree=tree)
    d.q, d.kt, d.vt, d.mask = c.q, c.kt, c.vt, c.mask
    slots = torch.full((3, 512), -1, dtype=torch.int32)
    table = d.cache.page_table.cpu()
    for b, L in enumerate(lens):
        p = torch.arange(L)
        slots[b, :L] = table[b, p // 16] * 16 + p % 16
    n = c.kq.shape[2]
    adapld.kv4_append(d.cache, c.kq.transpose(1, 2).contiguous(), c.vq.transpose(1, 2).contiguous(), slots[:, :n].contiguous().cuda())
    # (values of the grid may move to a finer scale, their values stay)
    again, _ = adapld.kv4_gather(d.cache, slots[:, :n].contiguous().cuda())
    assert torch.equal(again[0, :lens[0]], c.kq.transpose(1, 2)[0, :lens[0]])
    o2, l2 = d.run()
    for b, t in enumerate(counts):
        assert torch.equal(out[b, :t], o2[b, :t]) and torch.equal(lse[b, :, :t], l2[b, :, :t])


def test_verify_batch_mates_do_not_matter():
    c = Case([300, 20, 511, 0, 64, 450], 8, 2, 9, [9, 9, 2, 5, 9, 1], 16, 512, 31, tree="random")
    out, lse = c.run()
    lens, counts = list(c.lens), list(c.counts)
    for keep in (0, 4):
        c.lens = [n if b == keep else 17 for b, n in enumerate(lens)]
        c.lens[3] = 0 if keep != 3 else lens[3]
        c.lens = [min(a, b) for a, b in zip(c.lens, lens)]
        c.counts = [n if b == keep else 1 for b, n in enumerate(counts)]
        o2, l2 = c.run()
        t = counts[keep]
        assert torch.equal(out[keep, :t], o2[keep, :t]) and torch.equal(lse[keep, :, :t], l2[keep, :, :t])


def test_verify_leaves_other_rows():
    c = Case([100, 40], 4, 2, 6, [2, 0], 16, 128, 7, tree="random")
    out = torch.full((2, 6, 4, 128), 55.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((2, 4, 6), 55.0, device="cuda")
    c.run(out=out, lse=lse)
    assert (out[0, 2:] == 55).all() and (out[1] == 55).all() and (lse[0, :, 2:] == 55).all() and (lse[1] == 55).all()
    assert not (out[0, :2] == 55).any()
    o2, none = c.run(with_lse=False)
    assert none is None and torch.equal(o2[0, :2], out[0, :2])


def test_verify_bound_above_the_lengths():
    """A generous L_max gives the same attention (cut elsewhere)."""
    c = Case([200, 77], 8, 2, 5, [5, 5], 64, 256, 41, tree="random")
    out, lse = c.run()
    c.check(out, lse)
    cache = c.cache
    wide = torch.full((2, 700), -1, dtype=torch.int32, device="cuda")
    wide[:, :cache.page_table.shape[1]] = cache.page_table
    cache.page_table = wide
    for L_max in (3000, 700 * 64):
        out, lse = c.run(L_max=L_max)
        c.check(out, lse)
    # a bound below a length cuts the sequence there
    out, lse = c.run(L_max=100)
    c.check(out, lse, lens=[100, 77])


def test_verify_scale():
    c = Case([130], 4, 2, 3, [3], 16, 130, 43, tree="chain")
    out, lse = c.run(scale=0.25)
    c.check(out, lse, scale=0.25)


def test_verify_like_the_dense_cache():
    """The bf16 entry point on the values that the codes stand for."""
    c = Case([700, 33, 512], 8, 2, 20, [20, 3, 11], 32, 700, 47, tree="random", empty=0.0)
    out, lse = c.run()
    o2, l2 = adapld.tree_verify_attn(c.q, c.kq, c.vq, c.kt, c.vt, i32(c.lens), i32(c.counts), c.mask)
    for b, t in enumerate(c.counts):
        # both are within the bound of the exact result; outputs are averages of N(0, 1) values
        assert (out[b, :t].float() - o2[b, :t].float()).abs().max() <= 2 * 2.0 ** -8 * 5
        assert (lse[b, :, :t] - l2[b, :, :t]).abs().max() <= 1e-4


def test_offsets_beyond_32_bits():
    """Pages at the end of a pool whose arrays hold more than 4 GiB each."""
    page, Hkv = 256, 8
    n_pages = (5 << 30) // (page * Hkv * 64)
    cache = adapld.Kv4Cache.allocate(n_pages, page, Hkv, 1, 4)
    assert cache.k_codes.numel() > 1 << 32
    rng = np.random.default_rng(3)
    L = 700
    cache.page_table.copy_(i32([[n_pages - 1, 1, n_pages - 2, 0]]))
    k, v = (bf16(rng.standard_normal((1, L, Hkv, 128))).cuda() for _ in range(2))
    slots, granted = torch.empty((1, L), dtype=torch.int32, device="cuda"), None
    p = torch.arange(L, device="cuda")
    slots[0] = cache.page_table[0, p // page] * page + p % page
    adapld.kv4_append(cache, k, v, slots)
    kq, vq = adapld.kv4_gather(cache, slots)
    code, e = oracle.kv4_quantise(f64(k[0, 600, 5]))
    assert np.array_equal(f64(kq[0, 600, 5]), oracle.kv4_values(oracle.kv4_pack(code), e))
    q = bf16(rng.standard_normal((1, 1, 16, 128))).cuda()
    out, lse = adapld.tree_verify_attn_kv4(q, cache, i32([L]), i32([1]), L_max=L)
    z = torch.matmul(q.double().view(Hkv, 2, 128), kq[0].double().permute(1, 2, 0)) / math.sqrt(128)
    want = torch.matmul(z.softmax(-1), vq[0].double().transpose(0, 1)).view(1, 1, 16, 128)
    assert (out.double() - want).abs().max() < 2.0 ** -8 * 4
    assert (lse.view(-1).double() - z.logsumexp(-1).view(-1)).abs().max() < 1e-5


def test_long_context():
    """Lengths that take many splits, against float64 on the GPU."""
    L, Hkv, Hq, T, page = 40001, 2, 8, 3, 64
    c = Case([L], Hq, Hkv, T, [T], page, L, 53)
    out, lse = c.run()
    q = c.q[0].double().view(T, Hkv, 4, 128).permute(1, 2, 0, 3).reshape(Hkv, 4 * T, 128)
    z = torch.matmul(q, c.kq[0].double().transpose(1, 2)) / math.sqrt(128)
    want = torch.matmul(z.softmax(-1), c.vq[0].double()).view(Hq, T, 128).transpose(0, 1)
    spread = torch.matmul(z.softmax(-1), c.vq[0].double().abs()).view(Hq, T, 128).transpose(0, 1)
    assert ((out[0].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2 * DELTA) * spread).all()
    assert (lse[0].double() - z.logsumexp(-1).view(Hq, T)).abs().max() < 1e-4


# ------------------------------------------------------- streams, graphs, loop

def test_other_stream():
    c = Case([300, 200], 8, 2, 7, [7, 7], 16, 300, 61, tree="random")
    out, lse = c.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    o2, l2 = c.run(stream=s)
    s.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_graph_replays():
    """A captured iteration (pages, append, attention) replayed over new inputs
    in the same buffers, eager work between the replays."""
    B, Hkv, Hq, T, page, L0 = 3, 2, 8, 6, 16, 200
    c = Case([L0, L0 - 7, 30], Hq, Hkv, T, [T] * B, page, 512, 67, tree="chain")
    old, new = i32(c.lens), i32([n + T for n in c.lens])
    counts = i32(c.counts)
    n_pages = c.cache.n_pages
    free = adapld.Kv4Cache.allocate(8, page, Hkv, B, 1)
    cache = adapld.Kv4Cache(*(torch.cat((x, y)) for x, y in zip(
        (c.cache.k_codes, c.cache.k_scales, c.cache.v_codes, c.cache.v_scales),
        (free.k_codes, free.k_scales, free.v_codes, free.v_scales))), page_table=c.cache.page_table,
        free_pages=torch.full((n_pages + 8,), -1, dtype=torch.int32, device="cuda"),
        free_count=i32([8]), page_size=page)
    cache.free_pages[:8] = torch.arange(n_pages, n_pages + 8, device="cuda", dtype=torch.int32)
    left = i32([0])
    out = torch.zeros((B, T, Hq, 128), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((B, Hq, T), device="cuda")
    need = adapld.workspace_bytes(adapld.OP_TREE_VERIFY_ATTN_KV4, B, 512, 0, 0, T, Hq, Hkv, 128)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    slots = torch.zeros((B, T), dtype=torch.int32, device="cuda")
    granted = i32([0] * B)

    def step():
        adapld.page_map(cache, old, new, slot_map=slots, granted=granted, free_count_out=left)
        adapld.kv4_append(cache, c.kt, c.vt, slots)
        adapld.tree_verify_attn_kv4(c.q, cache, new, counts, L_max=512, out=out, lse=lse, ws=ws)

    step()
    torch.cuda.synchronize()
    first = (out.clone(), lse.clone(), slots.clone(), left.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    q0, kt0 = c.q.clone(), c.kt.clone()
    for rep in range(4):
        c.q.copy_(q0 * (1 + rep % 2))
        c.kt.copy_(kt0 * (1 + rep % 2))
        out.fill_(9.0)
        step()
        torch.cuda.synchronize()
        want = (out.clone(), lse.clone(), slots.clone(), left.clone())
        out.fill_(9.0)
        slots.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((out, lse, slots, left), want):
            assert torch.equal(a, b), rep
        if rep % 2 == 0:
            for a, b in zip(want, first):
                assert torch.equal(a, b), rep


def test_decoding_loop():
    """Iterations as a server runs them: the root's K/V appended, the tree
    verified, accepted, its kept nodes appended; checked against a dense copy."""
    rng = np.random.default_rng(71)
    B, Hkv, Hq, W, S, page, cap = 4, 2, 8, 3, 2, 16, 256
    T = W * (S + 1)
    cache = adapld.Kv4Cache.allocate(B * cap // page, page, Hkv, B, cap // page)
    dense_k = np.zeros((B, Hkv, cap, 128))
    dense_v = np.zeros_like(dense_k)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")

    def store(x_k, x_v, adds, rows=None):
        """Appends adds[b] rows (rows picks them) to sequence b."""
        nonlocal lens
        new = lens + i32(adds)
        n = max(adds)
        slots, granted = adapld.page_map(cache, lens, new, n)
        assert granted.tolist() == [1] * B
        adapld.kv4_append(cache, x_k, x_v, slots, rows=None if rows is None else rows[:, :n].contiguous())
        for b, a in enumerate(adds):
            L = int(lens[b])
            for i in range(a):
                r = i if rows is None else int(rows[b, i])
                for x, d in ((x_k, dense_k), (x_v, dense_v)):
                    code, e = oracle.kv4_quantise(f64(x[b, r]))
                    d[b, :, L + i] = oracle.kv4_values(oracle.kv4_pack(code), e)
        lens = new

    new_rows = lambda n: (bf16(rng.standard_normal((B, n, Hkv, 128))).cuda() for _ in range(2))  # noqa: E731
    store(*new_rows(40), [40, 1, 17, 33])   # prompts
    parent = np.array([-1 if u % (S + 1) == 0 else u - 1 for u in range(T)])
    depth = np.arange(T) % (S + 1)
    sees = np.array([[v // (S + 1) == u // (S + 1) and v <= u for v in range(T)] for u in range(T)])
    words = np.array([sum(1 << v for v in range(T) if sees[u, v]) for u in range(T)], dtype=np.int64)
    mask = torch.from_numpy(np.tile(words[None, :, None], (B, 1, 1))).cuda()
    for it in range(6):
        store(*new_rows(1), [1] * B)        # the root token of the iteration
        kt, vt = new_rows(T)
        q = bf16(rng.standard_normal((B, T, Hq, 128))).cuda()
        counts = [T, T - 2, 1, T]
        out, lse = adapld.tree_verify_attn_kv4(q, cache, lens, i32(counts), k_tree=kt, v_tree=vt, tree_mask=mask)
        L = lens.tolist()
        o, l, spread, _ = oracle.kv4_verify(f64(q), dense_k, dense_v, L, counts, f64(kt), f64(vt),
                                            np.tile(sees[None], (B, 1, 1)))
        for b, t in enumerate(counts):
            assert (np.abs(f64(out[b, :t]) - o[b, :t]) <= 2.0 ** -8 * np.abs(o[b, :t])
                    + (2.0 ** -8 + 2 * DELTA) * spread[b, :t]).all(), (it, b)
            assert np.abs(f64(lse[b, :, :t]) - l[b, :, :t]).max() < 1e-4
        token = rng.integers(0, 3, (B, T))
        target = rng.integers(0, 3, (B, T + 1))
        tile = lambda x: i32(np.tile(x[None], (B, 1)).tolist())  # noqa: E731
        n, nodes, _ = adapld.accept_greedy(i32(token.tolist()), tile(parent), tile(depth), i32(counts), mask,
                                           i32(target.tolist()), lens)
        adds = n.tolist()
        if max(adds):
            store(kt, vt, adds, rows=nodes)
    # every sequence ends: all pages are back
    adapld.page_map(cache, lens, torch.zeros_like(lens))
    assert int(cache.free_count) == cache.n_pages
    assert sorted(cache.free_pages.tolist()) == list(range(cache.n_pages))
