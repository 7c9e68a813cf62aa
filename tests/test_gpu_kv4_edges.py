"""The 4-bit cache's entry points where they can go wrong: page ids past one
register's worth of steps, logits that outgrow the exponent's range, pages that
are no pages of the pool, calls at once, buffers exchanged, the largest trees
and batches.  Bounds as in test_gpu_kv4.py, with each row's own logit error
where logits are large."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_05742_amd as adapld
from test_gpu_kv4 import DELTA, Case, _check_map, _fill, bf16, f64, i32

pytestmark = pytest.mark.gpu


def _check_loose(c, out, lse):
    """Case.check with the logits' error in the bound (for logits beyond 128)."""
    tree = (None, None, None) if c.kt is None else (f64(c.kt), f64(c.vt), c.sees)
    o, l, spread, reach = oracle.kv4_verify(f64(c.q), f64(c.kq), f64(c.vq), c.lens, c.counts, *tree)
    for b, t in enumerate(c.counts):
        n = c.lens[b] + t
        delta = reach[b, :, :t] * (2.0 ** -23 + 130 * 2.0 ** -24) + 2.0 ** -22 + n * 2.0 ** -28
        d = np.moveaxis(delta, 0, 1)[..., None]
        tol = 2.0 ** -8 * np.abs(o[b, :t]) + (2.0 ** -8 + 2 * d) * spread[b, :t]
        assert (np.abs(f64(out[b, :t]) - o[b, :t]) <= tol + 1e-30).all(), b
        assert (np.abs(f64(lse[b, :, :t]) - l[b, :, :t]) <= 2.0 ** -22 * np.abs(l[b, :, :t]) + delta).all(), b


@pytest.mark.parametrize("T, Hq, Hkv, tree", [(1, 4, 1, None), (7, 4, 1, "random"), (15, 4, 1, "chain"),
                                              (30, 4, 1, "random"), (70, 4, 1, "random")])
def test_logits_beyond_the_exponents_range(T, Hq, Hkv, tree):
    """Rows whose logits grow by hundreds after the first keys: weights relative
    to an early key overflow, and the step is done again."""
    c = Case([900, 333], Hq, Hkv, T, [T, max(T // 2, 1)], 16, 900, 83, tree=tree, wide=60.0)
    out, lse = c.run()
    assert torch.isfinite(out[0]).all() and torch.isfinite(lse[0]).all()
    _check_loose(c, out, lse)


@pytest.mark.parametrize("T, Hq, Hkv, lens", [
    (64, 2, 2, [100, 0, 65]), (33, 1, 1, [700]), (100, 4, 2, [0, 50, 64]), (256, 8, 1, [130]), (40, 16, 2, [64, 128]),
    (9, 64, 8, [70, 1]), (2, 8, 1, [31])])
def test_tree_shapes(T, Hq, Hkv, lens):
    """Two tree steps of independent waves, tiles of the tree alone, 2048 rows."""
    counts = [T if b % 2 == 0 else max(T - 5, 1) for b in range(len(lens))]
    c = Case(lens, Hq, Hkv, T, counts, 32, max(max(lens), 1), T, tree="random", empty=0.3)
    out, lse = c.run()
    c.check(out, lse)


def _gpu_reference(c, kq, vq, b, g):
    """float64 on the GPU for one (sequence, kv head): out [T, G, D], lse, spread."""
    G = c.q.shape[2] // c.Hkv
    T, L = c.counts[b], c.lens[b]
    k, v = kq[b, g, :L].double(), vq[b, g, :L].double()
    q = c.q[b, :T, g * G:(g + 1) * G].double()
    z = torch.matmul(q.reshape(T * G, 128), k.t()) / math.sqrt(128)
    if c.kt is not None:
        zt = torch.matmul(q.reshape(T * G, 128), c.kt[b, :T, g].double().t()) / math.sqrt(128)
        see = torch.from_numpy(c.sees[b, :T, :T]).cuda().repeat_interleave(G, 0)
        z = torch.cat((z, zt.masked_fill(~see, -math.inf)), 1)
        v = torch.cat((v, c.vt[b, :T, g].double()))
    p = z.softmax(-1)
    return (torch.matmul(p, v).view(T, G, 128), z.logsumexp(-1).view(T, G), torch.matmul(p, v.abs()).view(T, G, 128))


@pytest.mark.parametrize("T, Hq, Hkv, L", [(1, 32, 8, 20011), (8, 32, 8, 20011), (16, 32, 8, 17000), (20, 32, 8, 6007),
                                           (52, 32, 8, 10007)])
def test_long_splits(T, Hq, Hkv, L):
    """More steps of one wave than a register holds page ids for (16384, 8192 or
    4096 keys of a split), in batches that leave the context whole."""
    B = 32 if T < 52 else 16
    c = Case([L - 17 * b for b in range(B)], Hq, Hkv, T, [T] * B, 64, L, 89, tree="chain" if T > 1 else None)
    out, lse = c.run()
    for b, g in ((0, 0), (0, Hkv - 1), (B - 1, 3)):
        o, l, spread = _gpu_reference(c, c.kq, c.vq, b, g)
        G = Hq // Hkv
        got = out[b, :T, g * G:(g + 1) * G].double()
        assert ((got - o).abs() <= 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2 * DELTA) * spread).all(), (b, g)
        assert (lse[b, g * G:(g + 1) * G, :T].t().double() - l).abs().max() < 1e-4, (b, g)


def test_many_sequences():
    """Several rounds of workgroups; each sequence as if it were alone."""
    rng = np.random.default_rng(5)
    B = 300
    lens = rng.integers(0, 90, B).tolist()
    c = Case(lens, 8, 8, 2, [1 + b % 2 for b in range(B)], 16, 96, 97, tree="chain")
    out, lse = c.run()
    c.check(out, lse)


def test_pages_outside_the_pool():
    """A table entry that is no page of the pool spoils its own sequence only."""
    for T in (1, 30):
        c = Case([300, 290, 100], 8, 2, T, [T] * 3, 16, 300, 101, tree="chain")
        out, lse = c.run()
        good = (out.clone(), lse.clone())
        n = c.cache.n_pages
        for i, bad in enumerate((-1, n, (1 << 31) - 1, -(1 << 31))):
            c.cache.page_table[0, 2 * i] = bad
        out, lse = c.run()
        torch.cuda.synchronize()
        for b in (1, 2):
            assert torch.equal(out[b], good[0][b]) and torch.equal(lse[b], good[1][b])


def test_same_slot_twice():
    """Two rows for one slot: every stored byte is one of the two rows', and no
    other byte moves."""
    rng = np.random.default_rng(7)
    cache = adapld.Kv4Cache.allocate(3, 16, 2, 1, 1)
    _fill(cache, rng)
    k, v = bf16(rng.standard_normal((1, 2, 2, 128))).cuda(), bf16(rng.standard_normal((1, 2, 2, 128))).cuda()
    before = [t.clone() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    adapld.kv4_append(cache, k, v, i32([[20, 20]]))
    for t, old, x in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), before, (k, k, v, v)):
        code, e = oracle.kv4_quantise(f64(x[0]))
        want = oracle.kv4_pack(code) if t.shape[-1] == 64 else e
        got = t[1, :, 4].cpu().numpy()
        assert ((got == want[0]) | (got == want[1])).all()
        old[1, :, 4] = t[1, :, 4]
        assert torch.equal(t, old)


def test_two_calls_at_once():
    """Two batches on two streams over one pool, each with its own workspace."""
    a = Case([3000, 100], 8, 2, 5, [5, 5], 64, 3000, 103, tree="random")
    d = Case([777, 2500], 8, 2, 20, [20, 11], 64, 2600, 107, tree="random")
    want = [(o.clone(), l.clone()) for o, l in (a.run(), d.run())]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [(torch.zeros_like(o), torch.zeros_like(l)) for o, l in want]
    ws = [torch.empty(max(adapld.workspace_bytes(adapld.OP_TREE_VERIFY_ATTN_KV4, 2, c.L_max, 0, 0, c.T, 8, 2, 128), 16),
                      dtype=torch.uint8, device="cuda") for c in (a, d)]
    sizes = [(i32(c.lens), i32(c.counts)) for c in (a, d)]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, n, (o, l), w, s in zip((a, d), sizes, outs, ws, (s1, s2)):
            adapld.tree_verify_attn_kv4(c.q, c.cache, *n, k_tree=c.kt, v_tree=c.vt, tree_mask=c.mask, L_max=c.L_max,
                                        out=o, lse=l, ws=w, stream=s)
    torch.cuda.synchronize()
    for (o, l), (wo, wl), c in zip(outs, want, (a, d)):
        for b, t in enumerate(c.counts):
            assert torch.equal(o[b, :t], wo[b, :t]) and torch.equal(l[b, :, :t], wl[b, :, :t])


def test_exchanged_buffers_are_seen():
    """A field of the cache that is assigned replaces the marshalled buffer."""
    c = Case([64], 4, 2, 1, [1], 16, 64, 109)
    out, lse = c.run()
    old = c.cache.k_scales
    c.cache.k_scales = torch.full_like(old, 100)     # keys of size 2^-27: uniform weights
    flat, _ = c.run()
    mean = c.vq[0].double().mean(1)                  # [Hkv, D]
    for h in range(4):
        # weights 1/64 each are exact in bf16
        assert (flat[0, 0, h].double() - mean[h // 2]).abs().max() <= 2.0 ** -8 * mean.abs().max() + 1e-4
    c.cache.k_scales = old
    again, _ = c.run()
    assert torch.equal(out, again)
    with pytest.raises(adapld.AdapldError):
        c.cache.k_scales = old[:, :1]
        c.run()
    c.cache.k_scales = old.cpu()
    with pytest.raises(adapld.AdapldError):
        c.run()


def test_moved_buffers_are_seen():
    """A buffer whose memory is exchanged in place is marshalled again."""
    c = Case([64], 4, 2, 1, [1], 16, 64, 109)
    out, lse = c.run()
    for name in ("k_codes", "k_scales", "v_codes", "v_scales", "page_table"):
        t = getattr(c.cache, name)
        old = t.data
        t.data = old.clone()
        old.fill_(1)             # finite codes, page 1
        o2, l2 = c.run()
        assert torch.equal(out, o2) and torch.equal(lse, l2), name


def test_moved_stack_is_seen():
    cache = adapld.Kv4Cache.allocate(6, 16, 1, 2, 3)
    assert adapld.page_map(cache, i32([0, 0]), i32([16, 17]), 1)[0].tolist() == [[0], [16]]
    for t, v in ((cache.free_pages, [5, 4, 3, -1, -1, -1]), (cache.free_count, [3])):
        old = t.data
        t.data = i32(v)
        old.fill_(0)             # an empty stack of page 0
    slots, granted = adapld.page_map(cache, i32([16, 17]), i32([32, 33]), 17)
    assert granted.tolist() == [1, 1] and slots[0, :16].tolist() == list(range(48, 64))
    assert slots[1].tolist() == list(range(33, 48)) + [64, -1] and cache.free_count.tolist() == [1]
    with pytest.raises(adapld.AdapldError):
        cache.free_count = cache.free_count.long()
        adapld.page_map(cache, i32([32, 33]), i32([32, 33]), 1)


def test_own_buffers_belong_to_the_stream():
    """What a call on another stream makes for itself is of that stream: its
    fill comes before the kernel, and memory that it frees is not handed out on
    the current stream while the kernel is still to come."""
    c = Case([3000, 2000], 8, 2, 5, [5, 5], 64, 3000, 127, tree="random")
    want, want_lse = (t.clone() for t in c.run())
    slots = i32([[0, 5, 17]])
    k_want, v_want = (t.clone() for t in adapld.kv4_gather(c.cache, slots))
    lens, counts = i32(c.lens), i32(c.counts)
    need = adapld.workspace_bytes(adapld.OP_TREE_VERIFY_ATTN_KV4, 2, c.L_max, 0, 0, 5, 8, 2, 128)
    assert need > 0
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    out, lse = adapld.tree_verify_attn_kv4(c.q, c.cache, lens, counts, k_tree=c.kt, v_tree=c.vt, tree_mask=c.mask,
                                           L_max=c.L_max, stream=s)
    others = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (need, out.numel() * 2, lse.numel() * 4)]
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert all(bool((t == 7).all()) for t in others)
    torch.cuda._sleep(20_000_000)           # a fill on the current stream would come late
    k, v = adapld.kv4_gather(c.cache, slots, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(k, k_want) and torch.equal(v, v_want)


def test_refusals_of_gpu_tensors():
    c = Case([64, 30], 4, 2, 2, [2, 2], 16, 64, 113, tree="chain")
    for kw in (dict(tree_mask=None), dict(k_tree=c.kt.half()), dict(v_tree=c.vt[:, :1]), dict(L_max=10 ** 6),
               dict(L_max=0), dict(scale=0.0), dict(out=torch.zeros((2, 2, 4, 64), device="cuda")),
               dict(tree_mask=c.mask[:1]), dict(lse=torch.zeros((2, 4, 2), dtype=torch.float64, device="cuda"))):
        with pytest.raises(adapld.AdapldError):
            c.run(**kw)
    q = c.q
    for bad in (q[..., :64].contiguous(), q[:1], q.transpose(1, 2)):
        c.q = bad
        with pytest.raises(adapld.AdapldError):
            c.run()
    slots = i32([[0, 1], [2, 3]])
    with pytest.raises(adapld.AdapldError):
        adapld.kv4_append(c.cache, c.kt, c.vt, slots.long())
    with pytest.raises(adapld.AdapldError):
        adapld.kv4_append(c.cache, c.kt, c.vt, i32([[0, 1, 2], [3, 4, 5]]))       # more slots than rows
    with pytest.raises(adapld.AdapldError):
        adapld.kv4_append(c.cache, c.kt, c.vt, slots, rows=i32([[0, 1]]))
    with pytest.raises(adapld.AdapldError):
        adapld.kv4_gather(c.cache, slots, k_out=torch.zeros((2, 2, 2, 128), device="cuda"))
    with pytest.raises(adapld.AdapldError):
        adapld.page_map(c.cache, i32([1]), i32([2, 2]), 1)
    with pytest.raises(TypeError):
        adapld.page_map(c.cache, [1, 1], [2, 2], 1)


@pytest.mark.parametrize("B, N, in_place", [(1024, 9, False), (1025, 9, False), (1024, 9, True), (3, 6000, True),
                                            (2, 4096, False), (700, 33, False), (1, 1, True), (90, 6000, False)])
def test_page_map_every_way_to_the_slots(B, N, in_place):
    """Slots by the first workgroup, by others beside it, by a second launch,
    with sequences that give back what others take."""
    rng = np.random.default_rng(B + N)
    page, max_pages = 16, 6000 // 16 + 4 if N > 1000 else 8
    top = max_pages * page
    old = rng.integers(0, top // 2 + 1, B)
    new = np.where(rng.random(B) < 0.4, rng.integers(0, old + 1), np.minimum(old + rng.integers(0, N + 1, B), top))
    held = -(-old // page)
    used = int(held.sum())
    spare = max(int(np.maximum(-(-new // page) - held, 0).sum()) // 2, 1)   # the rest comes from those that end
    ids = rng.permutation(used + spare)
    table = np.full((B, max_pages), -1)
    at = 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    free = np.full(used + spare, -5)
    free[:spare] = ids[used:]
    _check_map(old.tolist(), new.tolist(), page, table.tolist(), free.tolist(), spare, N, in_place)
