"""Attention weights of many stacked rows against float64: prompt chunks of batches, more
rows than fit LDS at a time, rows that give nothing among them.

A stacked row is a new row's query head; N * Hq / Hkv of them share a kv head's keys.
Above 256 they pass through a ring in LDS against 256 or 128 keys a workgroup, whichever
takes the fewer rounds over the CUs, 2048 at a time; each test says which it is meant to
reach.  Bounds as in test_gpu_kv8_evict.py.
"""
import math

import numpy as np
import pytest
import torch

import paper_2606_05742_amd as adapld
from test_gpu_kv4 import bf16, i32
from test_gpu_kv8 import make_cache, values

pytestmark = pytest.mark.gpu


def check_rows(new, add, Hq, Hkv, T, page, N=None, rows=None, silent=None, seed=0):
    """Sequence b goes from new[b] - add[b] to new[b] tokens; silent(b, i, h) says which
    (sequence, new row, head) has no log-sum-exp."""
    rng = np.random.default_rng(seed + T)
    B, G, L, scale = len(new), Hq // Hkv, max(new), 1.0 / math.sqrt(128)
    N = T if N is None else N
    old = [n - a for n, a in zip(new, add)]
    cache, table = make_cache(new, page, Hkv, rng)
    k, v = (bf16(rng.standard_normal((B, L, Hkv, 128))).cuda() for _ in range(2))
    adapld.kv8_append(cache, k, v, i32([0] * B), i32(new))
    q = bf16(rng.standard_normal((B, T, Hq, 128))).cuda()
    lse = torch.full((B, Hq, T), math.nan, device="cuda")      # of queries that no row picks
    w = torch.from_numpy(rng.random((B, Hkv, L + 3)).astype(np.float32)).cuda()
    p = torch.full((B, Hkv, L + 3), -5, dtype=torch.int32, device="cuda")
    first = [1000 * b + 7 for b in range(B)]

    # the logits of a kv head's rows [n * G, new[b]], and which keys they see
    def logits(b, g):
        keys = values(cache.k_codes[table[b, :-(-new[b] // page)], g], cache.k_scales[table[b, :-(-new[b] // page)], g])
        keys = keys.reshape(-1, 128)[:new[b]].double()
        u = torch.arange(add[b]) if rows is None else torch.tensor(rows[b][:add[b]])
        ok = (u >= 0) & (u < T)
        x = q[b, torch.where(ok, u, 0).cuda(), g * G:(g + 1) * G].double().reshape(-1, 128)
        z, size = torch.matmul(x, keys.t()) * scale, torch.matmul(x.abs(), keys.abs().t()) * scale
        sees = torch.arange(new[b], device="cuda") <= (old[b] + torch.arange(add[b], device="cuda"))[:, None]
        return u, ok, z, size, sees.repeat_interleave(G, 0)

    for b in range(B):
        for g in range(Hkv):
            u, ok, z, _, sees = logits(b, g)
            s = z.masked_fill(~sees, -math.inf).logsumexp(-1).view(add[b], G).float()
            for i in range(add[b]):
                if ok[i]:
                    lse[b, g * G:(g + 1) * G, int(u[i])] = s[i]
        for i in range(add[b] if silent else 0):
            for h in range(Hq):
                if silent(b, i, h):
                    lse[b, h, i] = -math.inf if (i + h) % 2 else math.nan
    call = lambda out: adapld.kv8_attn_weights(cache, q, lse, i32(old), i32(new), i32(first), w, p, N=N, L_max=L,  # noqa: E731
                                               rows=None if rows is None else i32(rows), weights_out=out)[0]
    got = call(torch.full_like(w, 7.5))
    torch.cuda.synchronize()
    for b in range(B):
        for g in range(Hkv):
            u, ok, z, size, sees = logits(b, g)
            own = lse[b, g * G:(g + 1) * G][:, torch.where(ok, u, 0).cuda()].t().reshape(-1).double()
            gives = ok.cuda().repeat_interleave(G) & torch.isfinite(own)
            part = sees & gives[:, None]
            want = torch.where(part, (z - own[:, None]).exp(), 0.0).sum(0)
            before = torch.where(torch.arange(new[b], device="cuda") < old[b], w[b, g, :new[b]].double(), 0.0)
            reach = torch.where(part, size, 0.0).max()
            top = torch.where(gives, own.abs(), 0.0).max()
            rel = reach * (2.0 ** -23 + 130 * 2.0 ** -24) + 2.0 ** -22 * (reach + top) + 2.0 ** -22 + (add[b] * G + 1) * 2.0 ** -24
            tol = rel * want + 2.0 ** -23 * (want + before) + add[b] * G * 2.0 ** -126
            assert ((got[b, g, :new[b]].double() - want - before).abs() <= tol).all(), (b, g)
            assert (got[b, g, new[b]:] == 7.5).all()
            assert (p[b, g, :old[b]] == -5).all() and (p[b, g, new[b]:] == -5).all()
            assert p[b, g, old[b]:new[b]].tolist() == [first[b] + i for i in range(add[b])]
    # the same bits again, and in place
    assert torch.equal(call(torch.full_like(w, 7.5)), got)
    now = call(w)
    assert now is w
    for b in range(B):
        assert torch.equal(w[b, :, :new[b]], got[b, :, :new[b]])


@pytest.mark.parametrize("page", [16, 64])
def test_prompt_chunk_of_a_batch(page):
    """1792 stacked rows; 256 keys a workgroup."""
    check_rows([4091, 3000, 517, 258], [256, 201, 256, 1], 28, 4, 256, page)


def test_accepted_rows_of_a_batch():
    """1400 stacked rows of queries in any order, some twice, some that are none; 256 keys a
    workgroup."""
    rng = np.random.default_rng(8)
    rows = rng.integers(-1, 257, (4, 200)).tolist()
    rows[1] = rng.permutation(256)[:200].tolist()
    rows[2][:40], rows[3][5] = [2 ** 31 - 1] * 40, -2 ** 31
    check_rows([4091, 700, 2049, 1000], [200, 131, 200, 33], 28, 4, 256, 32, N=200, rows=rows)


def test_more_rows_than_fit_at_a_time():
    """5020 stacked rows, 2048, 2048 and 924; 128 keys a workgroup."""
    check_rows([701, 260], [251, 130], 20, 1, 251, 16)


def test_more_rows_than_fit_at_a_time_of_a_batch():
    """4096 stacked rows in two parts; 256 keys a workgroup."""
    check_rows([1999, 1000, 257, 1990, 256, 300, 1537, 640], [256, 255, 256, 129, 256, 1, 200, 140], 64, 4, 256, 64)


@pytest.mark.parametrize("Hkv, B, L", [(1, 4, 700), (4, 8, 1999)])
def test_parts_of_the_rows_give_nothing(Hkv, B, L):
    """4096 stacked rows, 128 and 256 keys a workgroup: the first 2048 give nothing, the
    others, all of them, or one head here and there."""
    silent = lambda b, i, h: (i < 128, i >= 128, True, (7 * i + 5 * h + b) % 3 > 0)[b % 4]  # noqa: E731
    check_rows([L - 5 * b for b in range(B)], [256] * B, 16 * Hkv, Hkv, 256, 32, silent=silent)


@pytest.mark.parametrize("T, Hq, Hkv, L", [(1, 8, 2, 700), (16, 8, 2, 700), (40, 8, 2, 3000), (100, 8, 2, 700), (256, 28, 4, 1000)])
def test_batch_mates_do_not_matter(T, Hq, Hkv, L):
    """A sequence's bits stay where the others get shorter or add no rows."""
    rng = np.random.default_rng(T)
    new = [L - 7, L, L // 2 + T]
    cache, _ = make_cache(new, 32, Hkv, rng)
    k, v = (bf16(rng.standard_normal((3, L, Hkv, 128))).cuda() for _ in range(2))
    adapld.kv8_append(cache, k, v, i32([0] * 3), i32(new))
    q = bf16(rng.standard_normal((3, T, Hq, 128))).cuda()
    lse = torch.from_numpy(rng.random((3, Hq, T)).astype(np.float32) * 3 + 5).cuda()
    w, p = torch.rand((3, Hkv, L), device="cuda"), torch.zeros((3, Hkv, L), dtype=torch.int32, device="cuda")
    call = lambda old, new: adapld.kv8_attn_weights(cache, q, lse, i32(old), i32(new), i32([0] * 3), w, p,  # noqa: E731
                                                    weights_out=torch.zeros_like(w))[0]
    want = call([n - T for n in new], new)
    for b in range(3):
        got = call([n - T if x == b else 3 for x, n in enumerate(new)], [n if x == b else 3 + x for x, n in enumerate(new)])
        assert torch.equal(got[b], want[b])
