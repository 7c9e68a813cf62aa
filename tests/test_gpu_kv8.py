"""The paged 8-bit K/V cache on the GPU: rows and the verify attention against the
float64 reference.

Stored bytes are exact.  The attention's bounds are those of test_gpu_kv4.py: the
kernels, the products' operands (exact bf16 values) and the rounding of weights
are the same.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_05742_amd as adapld
from test_gpu_kv4 import CASES, DELTA, PAGES, Case, bf16, f64, i32

pytestmark = pytest.mark.gpu


def arrays(cache):
    return [t.cpu().numpy().copy() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]


def fill(cache, rng):
    """Bytes of any kind in rows and scales."""
    for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        t.copy_(torch.from_numpy(rng.integers(0, 256, t.shape, dtype=np.uint8)))


def make_cache(lens, page, Hkv, rng, max_pages=None, spare=2):
    """A cache with a table of pages in random order for `lens`, garbage in it."""
    max_pages = max(max(-(-n // page) for n in lens), 1) if max_pages is None else max_pages
    held = [-(-max(n, 0) // page) for n in lens]
    n_pages = sum(held) + spare
    ids = rng.permutation(n_pages)
    table = np.full((len(lens), max_pages), -1)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = ids[at:at + n]
        at += n
    cache = adapld.Kv8Cache.allocate(n_pages, page, Hkv, len(lens), max_pages)
    fill(cache, rng)
    cache.page_table.copy_(i32(table))
    return cache, table


def values(codes, scales):
    """float32 values on the GPU of codes [..., page, D]."""
    e = (scales.to(torch.int32) << 23).view(torch.float32).repeat_interleave(16, -1)
    return codes.view(torch.float8_e4m3fn).float() * e.unsqueeze(-1)


# ----------------------------------------------------------------------- rows

def check_append(k, v, old, new, page, rows=None, N=None, before=(), table_of=None, seed=11):
    """Every byte of the pool is the reference's after each of the appends."""
    rng = np.random.default_rng(seed)
    cache, table = make_cache([max(n, 0) for n in (table_of or new)], page, k.shape[2], rng)
    want = arrays(cache)
    for kk, vv, o, n, r, m in (*before, (k, v, old, new, rows, N)):
        oracle.kv8_append(f64(kk), f64(vv), o, n, table, page, want, r, m)
        adapld.kv8_append(cache, kk.cuda(), vv.cuda(), i32(o), i32(n), rows=None if r is None else i32(r), N=m)
        for got, w in zip(arrays(cache), want):
            assert np.array_equal(got, w)
    return cache, table


def rows_of(rng, B, n, Hkv, spread=6):
    x = rng.standard_normal((B, n, Hkv, 128)) * np.exp2(rng.integers(-spread, spread + 1, (B, n, Hkv, 1)))
    return bf16(x), bf16(rng.standard_normal((B, n, Hkv, 128)))


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("B, N, Hkv", [(1, 1, 1), (2, 15, 3), (3, 37, 8), (1, 130, 2)])
def test_append(page, B, N, Hkv):
    """A first part, then rows behind it that move the blocks' scales."""
    rng = np.random.default_rng(page + B + N)
    first = rng.integers(0, 40, B)
    add = np.array([max(1, N - 3 * b) for b in range(B)])
    pre = (*rows_of(rng, B, max(int(first.max()), 1), Hkv), [0] * B, first.tolist(), None, None)
    check_append(*rows_of(rng, B, N, Hkv, 20), first.tolist(), (first + add).tolist(), page, before=[pre])


def test_append_one_token_at_a_time():
    """A block takes its tokens one by one, each larger than the last, then smaller."""
    rng = np.random.default_rng(5)
    steps = []
    for i in range(40):
        x = bf16(rng.standard_normal((2, 1, 2, 128)) * 2.0 ** (i if i < 20 else 40 - i))
        steps.append((x, bf16(rng.standard_normal((2, 1, 2, 128))), [i, i + 3], [i + 1, i + 4], None, None))
    pre = (*rows_of(rng, 2, 3, 2), [0, 0], [0, 3], None, None)
    check_append(*steps[-1][:4], 16, before=[pre, *steps[:-1]], table_of=[40, 43])


def test_append_rows_and_bounds():
    """Rows picked from the source (one twice), rows outside it, lengths that shrink,
    stay, run past the capacity or past N, pages outside the pool."""
    rng = np.random.default_rng(21)
    k, v = rows_of(rng, 6, 9, 2)
    rows = [[8, 0, 3, 3], [4, 9, -1, 1 << 30], [0, 1, 2, 3], [1, 2, 3, 4], [5, 6, 7, 8], [0, 2, 4, 6]]
    old, new = [5, 30, 20, 17, 46, -4], [9, 33, 12, 17, 99, 3]
    check_append(k, v, old, new, 16, rows=rows, table_of=[48] * 6)
    check_append(k, v, [0, 3, 40, 2, 1, 7], [9, 9, 44, 3, 1, 30], 32, N=2, table_of=[48] * 6)
    cache, table = make_cache([64, 64], 16, 2, rng)
    want = arrays(cache)
    for i, bad in enumerate((-1, cache.n_pages, (1 << 31) - 1, -(1 << 31))):
        table[0, i] = bad
    cache.page_table.copy_(i32(table))
    k, v = rows_of(rng, 2, 50, 2)
    adapld.kv8_append(cache, k.cuda(), v.cuda(), i32([3, 3]), i32([53, 53]))
    oracle.kv8_append(f64(k), f64(v), [3, 3], [53, 53], table, 16, want)
    for got, w in zip(arrays(cache), want):
        assert np.array_equal(got, w)


def test_append_special_values():
    """Zeros, signed zeros, ties, the bounds of the scale, subnormals, values that no
    scale holds, infinities and NaN: each changes its own code alone."""
    rng = np.random.default_rng(23)
    x = np.zeros((1, 10 * 16, 1, 128), np.float32)
    put = lambda i, val: x.__setitem__((0, 16 * i, 0, slice(0, len(val))), val)  # noqa: E731
    x[0, 0, 0, 0] = -0.0
    put(1, [448.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, -(2.0 ** -9), 432.0, 27.0])
    put(2, [450.0, 464.0, 1.0])
    put(3, (rng.standard_normal(128) * 2.0 ** -130).tolist())
    put(4, [3.3895314e38, -3.3895314e38, 2.9e38, 1e38, 1.0])
    put(5, [math.inf, -math.inf, 3.0, 1e-3])
    put(6, [math.nan, 3.0, 1e-3, -math.nan])
    put(7, np.exp2(rng.integers(-60, 60, 128)).tolist())
    x[0, 16 * 8:16 * 9, 0] = math.inf
    x[0, 16 * 9:, 0] = rng.standard_normal((16, 128)) * 2.0 ** -117
    t = bf16(x)
    check_append(t, -t, [0], [160], 16)
    # and on top of older rows
    old = bf16(rng.standard_normal((1, 7, 1, 128)))
    for i in range(8):
        y = t[:, 16 * i:16 * i + 2]
        check_append(y, -y, [7], [9], 32, before=[(old, old, [0], [7], None, None)], table_of=[32])


@pytest.mark.parametrize("e", [10, 11, 100, 127, 245, 246])
def test_every_code(e):
    """All codes of a block's scale are read as their values, and rounded again when
    the scale rises by every number of steps that leaves something."""
    code = np.arange(256, dtype=np.uint8)
    code[[127, 255]] = 0
    for up in (1, 2, 5, 9, 10, 15, 17):
        if e + up > 246:
            continue
        cache = adapld.Kv8Cache.allocate(1, 16, 1, 1, 1)
        cache.page_table.fill_(0)
        for c, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
            c[0, 0, :2] = torch.from_numpy(code.reshape(2, 128)).cuda()
            s.fill_(e)
        want = arrays(cache)
        top = np.zeros((1, 1, 1, 128))
        top[..., 3] = 448.0 * 2.0 ** (e + up - 127)
        oracle.kv8_append(top, -top, [2], [3], [[0]], 16, want)
        assert want[1][0, 0, 0] == e + up
        adapld.kv8_append(cache, bf16(top).cuda(), bf16(-top).cuda(), i32([2]), i32([3]))
        for got, w in zip(arrays(cache), want):
            assert np.array_equal(got[:, :, :3] if got.ndim == 4 else got, w[:, :, :3] if w.ndim == 4 else w)


# ------------------------------------------------------------------ attention

class Case8(Case):
    """A cache filled through append, with garbage in every row and scale that no
    sequence owns."""

    def __init__(self, lens, Hq, Hkv, T, counts, page, L_max, seed, tree=None, empty=0.2, wide=1.0):
        super().__init__([0] * len(lens), Hq, Hkv, T, counts, page, L_max, seed, tree, empty, wide)
        rng = np.random.default_rng(seed + 1000)
        self.lens = lens
        B, Lc = len(lens), max(max(lens), 1)
        self.cache, self.table = make_cache([max(n, 0) for n in lens], page, Hkv, rng, -(-L_max // page) + 1)
        k = bf16(rng.standard_normal((B, Lc, Hkv, 128)) * wide).cuda()
        v = bf16(rng.standard_normal((B, Lc, Hkv, 128))).cuda()
        adapld.kv8_append(self.cache, k, v, i32([0] * B), i32(lens))
        self.read()

    def read(self):
        """kq, vq [B, Hkv, Lc, D]: the values that the codes stand for (zeros behind
        a sequence)."""
        B, Lc = len(self.lens), max(max(self.lens), 1)
        t = self.cache.page_table.long()
        n = torch.tensor([max(x, 0) for x in self.lens], device="cuda")
        live = torch.arange(t.shape[1] * self.page, device="cuda") < n[:, None]
        for name, c, s in (("kq", self.cache.k_codes, self.cache.k_scales), ("vq", self.cache.v_codes, self.cache.v_scales)):
            x = values(c[t.clamp(min=0)], s[t.clamp(min=0)]).transpose(1, 2).reshape(B, self.Hkv, -1, 128)
            x = torch.where(live[:, None, :, None], x, 0.0)[:, :, :Lc].contiguous()
            setattr(self, name, x.to(torch.bfloat16))
            assert torch.equal(getattr(self, name).float(), x)

    def run(self, **kw):
        a = dict(k_tree=self.kt, v_tree=self.vt, tree_mask=self.mask, L_max=self.L_max) | kw
        return adapld.tree_verify_attn_kv8(self.q, self.cache, i32(self.lens), i32(self.counts), **a)


@pytest.mark.parametrize("name", sorted(CASES))
def test_verify(name):
    c = Case8(seed=len(name), **CASES[name])
    out, lse = c.run()
    c.check(out, lse)


@pytest.mark.parametrize("T, Hq, Hkv, tree", [(1, 8, 2, None), (7, 8, 2, "random"), (16, 8, 2, "chain"),
                                              (40, 8, 2, "random"), (70, 16, 2, "random")])
@pytest.mark.parametrize("page", PAGES)
def test_verify_pages(T, Hq, Hkv, tree, page):
    """Every page size gives the same bits."""
    lens, counts = [333, 64, 500], [T, max(T // 2, 1), T]
    c, d = (Case8(lens, Hq, Hkv, T, counts, p, 512, 5, tree=tree) for p in (page, 16))
    d.q, d.kt, d.vt, d.mask, d.sees = c.q, c.kt, c.vt, c.mask, c.sees
    adapld.kv8_append(d.cache, c.kq.transpose(1, 2).contiguous(), c.vq.transpose(1, 2).contiguous(), i32([0] * 3), i32(lens))
    d.read()
    assert torch.equal(c.kq, d.kq) and torch.equal(c.vq, d.vq)
    out, lse = c.run()
    o2, l2 = d.run()
    c.check(out, lse)
    for b, t in enumerate(counts):
        assert torch.equal(out[b, :t], o2[b, :t]) and torch.equal(lse[b, :, :t], l2[b, :, :t])


def test_verify_leaves_other_rows():
    c = Case8([100, 40], 4, 2, 6, [2, 0], 16, 128, 7, tree="random")
    out = torch.full((2, 6, 4, 128), 55.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((2, 4, 6), 55.0, device="cuda")
    c.run(out=out, lse=lse)
    assert (out[0, 2:] == 55).all() and (out[1] == 55).all() and (lse[0, :, 2:] == 55).all() and (lse[1] == 55).all()
    assert not (out[0, :2] == 55).any()
    o2, none = c.run(with_lse=False)
    assert none is None and torch.equal(o2[0, :2], out[0, :2])


def test_verify_batch_mates_do_not_matter():
    c = Case8([300, 20, 511, 0, 64, 450], 8, 2, 9, [9, 9, 2, 5, 9, 1], 16, 512, 31, tree="random")
    out, lse = c.run()
    lens, counts = list(c.lens), list(c.counts)
    for keep in (0, 4):
        c.lens = [n if b == keep else min(n, 17) for b, n in enumerate(lens)]
        c.counts = [n if b == keep else 1 for b, n in enumerate(counts)]
        o2, l2 = c.run()
        t = counts[keep]
        assert torch.equal(out[keep, :t], o2[keep, :t]) and torch.equal(lse[keep, :, :t], l2[keep, :, :t])


def test_verify_like_the_dense_cache():
    """The bf16 entry point on the values that the codes stand for."""
    c = Case8([700, 33, 512], 8, 2, 20, [20, 3, 11], 32, 700, 47, tree="random", empty=0.0)
    out, lse = c.run()
    o2, l2 = adapld.tree_verify_attn(c.q, c.kq, c.vq, c.kt, c.vt, i32(c.lens), i32(c.counts), c.mask)
    for b, t in enumerate(c.counts):
        # both are within the bound of the exact result; outputs are averages of N(0, 1) values
        assert (out[b, :t].float() - o2[b, :t].float()).abs().max() <= 2 * 2.0 ** -8 * 5
        assert (lse[b, :, :t] - l2[b, :, :t]).abs().max() <= 1e-4


@pytest.mark.parametrize("T, Hq, Hkv, L", [(1, 32, 8, 20011), (8, 32, 8, 20011), (16, 32, 8, 17000), (52, 32, 8, 10007)])
def test_long_splits(T, Hq, Hkv, L):
    """More steps of one wave than a register holds page ids for, against float64."""
    B = 32 if T < 52 else 16
    check_heads(Case8([L - 17 * b for b in range(B)], Hq, Hkv, T, [T] * B, 64, L, 89, tree="chain" if T > 1 else None))


@pytest.mark.parametrize("T", [1, 8, 16])
def test_long_contexts_of_many_sequences(T):
    """The same for workgroups of four waves."""
    check_heads(Case8([9001 - 17 * b for b in range(33)], 32, 8, T, [T] * 33, 64, 9001, 97, tree="chain" if T > 1 else None))


@pytest.mark.parametrize("T, Hq, tree", [(1, 8, None), (1, 60, None), (4, 16, "random"), (7, 16, "random"),
                                         (15, 16, "random"), (16, 16, "chain")])
def test_many_short_sequences(T, Hq, tree):
    """More workgroups than CUs, which then have four waves."""
    lens = [(37 * b) % 91 for b in range(66)] + [0, 257, 511, 640]
    c = Case8(lens, Hq, 4, T, [T - b % min(T, 3) for b in range(70)], 16, 640, 53, tree=tree)
    out, lse = c.run()
    c.check(out, lse)


def check_heads(c):
    """Some heads of a case against float64."""
    out, lse = c.run()
    B, T, Hq, _ = c.q.shape
    Hkv, L = c.kq.shape[1], c.L_max
    G = Hq // Hkv
    for b, g in ((0, 0), (0, Hkv - 1), (B - 1, 3)):
        n = c.lens[b]
        k, v = c.kq[b, g, :n].double(), c.vq[b, g, :n].double()
        q = c.q[b, :T, g * G:(g + 1) * G].double().reshape(T * G, 128)
        z = torch.matmul(q, k.t()) / math.sqrt(128)
        if c.kt is not None:
            zt = torch.matmul(q, c.kt[b, :T, g].double().t()) / math.sqrt(128)
            see = torch.from_numpy(c.sees[b]).cuda().repeat_interleave(G, 0)
            z = torch.cat((z, zt.masked_fill(~see, -math.inf)), 1)
            v = torch.cat((v, c.vt[b, :T, g].double()))
        p = z.softmax(-1)
        o, spread = torch.matmul(p, v).view(T, G, 128), torch.matmul(p, v.abs()).view(T, G, 128)
        got = out[b, :T, g * G:(g + 1) * G].double()
        assert ((got - o).abs() <= 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2 * DELTA) * spread).all(), (b, g)
        assert (lse[b, g * G:(g + 1) * G, :T].t().double() - z.logsumexp(-1).view(T, G)).abs().max() < 1e-4, (b, g)


def test_offsets_beyond_32_bits():
    """Pages at the end of a pool whose arrays hold more than 4 GiB each."""
    page, Hkv = 256, 8
    n_pages = (5 << 30) // (page * Hkv * 128)
    cache = adapld.Kv8Cache.allocate(n_pages, page, Hkv, 1, 4)
    assert cache.k_codes.numel() > 1 << 32
    rng = np.random.default_rng(3)
    L = 700
    table = [n_pages - 1, 1, n_pages - 2, 0]
    cache.page_table.copy_(i32([table]))
    k, v = (bf16(rng.standard_normal((1, L, Hkv, 128))).cuda() for _ in range(2))
    adapld.kv8_append(cache, k, v, i32([0]), i32([L]))
    kq, vq = (values(c[table], s[table]).transpose(0, 1).reshape(Hkv, -1, 128)[:, :L].double() for c, s in (
        (cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)))
    block = f64(k[0, 592:608, 5])
    assert np.array_equal(f64(kq[5, 592:608]), oracle.kv8_values(oracle.kv8_codes(block, oracle.kv8_exponent(block)),
                                                                 oracle.kv8_exponent(block)))
    q = bf16(rng.standard_normal((1, 1, 16, 128))).cuda()
    out, lse = adapld.tree_verify_attn_kv8(q, cache, i32([L]), i32([1]), L_max=L)
    z = torch.matmul(q.double().view(Hkv, 2, 128), kq.transpose(1, 2)) / math.sqrt(128)
    want = torch.matmul(z.softmax(-1), vq).view(1, 1, 16, 128)
    assert (out.double() - want).abs().max() < 2.0 ** -8 * 4
    assert (lse.view(-1).double() - z.logsumexp(-1).view(-1)).abs().max() < 1e-5


def test_pages_outside_the_pool():
    """A table entry that is no page of the pool spoils its own sequence only."""
    for T in (1, 30):
        c = Case8([300, 290, 100], 8, 2, T, [T] * 3, 16, 300, 101, tree="chain")
        out, lse = c.run()
        for i, bad in enumerate((-1, c.cache.n_pages, (1 << 31) - 1, -(1 << 31))):
            c.cache.page_table[0, 2 * i] = bad
        o2, l2 = c.run()
        torch.cuda.synchronize()
        for b in (1, 2):
            assert torch.equal(out[b], o2[b]) and torch.equal(lse[b], l2[b])


def test_other_stream():
    c = Case8([300, 200], 8, 2, 7, [7, 7], 16, 300, 61, tree="random")
    out, lse = c.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    o2, l2 = c.run(stream=s)
    s.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2)
