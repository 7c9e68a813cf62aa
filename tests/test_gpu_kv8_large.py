"""The 8-bit cache's larger calls on the GPU: prompts whose rows are streamed into it,
evictions in one launch from more slots than threads hold, the attention of a chunk of a
prompt.  Rows and evictions are exact, byte for byte; the attention's bounds are those of
test_gpu_kv4.py.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2606_05742_amd as adapld
from test_gpu_kv4 import i32
from test_gpu_kv8 import Case8, arrays, check_append, check_heads, make_cache, rows_of
from test_gpu_kv8_evict import check_evict

pytestmark = pytest.mark.gpu


# -------------------------------------------------- above 65536 rows of K and of V

@pytest.mark.parametrize("page", [16, 64, 256])
def test_append_prompts(page):
    """Prompts of a batch, behind rows that fill a part of a block, with scales that move and
    values that are not finite."""
    rng = np.random.default_rng(page)
    B, N, Hkv = 5, 2003, 8
    k, v = rows_of(rng, B, N, Hkv, 20)
    k[0, 100:200:7, 2, 5], v[1, ::333, 7, 127], v[2, 40, 0] = math.inf, math.nan, -math.inf
    k[3, 1, 4, 9] = 3.3e38
    old = [0, 5, 16, 31, 7]
    pre = (*rows_of(rng, B, 31, Hkv), [0] * B, old, None, None)
    check_append(k, v, old, [o + n for o, n in zip(old, (2003, 2000, 1777, 3, 2001))], page, before=[pre])


def test_append_many_picked_rows():
    """Rows in any order, some twice, some outside the source, lengths beyond N and the
    capacity."""
    rng = np.random.default_rng(2)
    B, n_src, N, Hkv = 3, 2600, 3000, 8
    k, v = rows_of(rng, B, n_src, Hkv, 12)
    rows = rng.integers(-1, n_src + 1, (B, N)).tolist()
    rows[0][7], rows[1][8] = 2 ** 31 - 1, -2 ** 31
    check_append(k, v, [0, 9, 500], [4000, 2900, 3100], 32, rows=rows, table_of=[3040, 2900, 3072])


# ----------------------------------- at most 64 rows move, more than 8192 slots a kv head

KINDS = {"distinct": None, "few values": lambda r, s: r.integers(0, 3, s) / 2, "all equal": lambda r, s: np.full(s, 0.5)}


@pytest.mark.parametrize("weights", sorted(KINDS))
@pytest.mark.parametrize("lens, budget, recent", [([9000, 8961], 8960, 17), ([16384, 16383, 5], 16320, 0),
                                                  ([16417, 16390], 16384, 256), ([20000, 64, 16500], 64, 9),
                                                  ([33000], 32944, 20)])
def test_evict_in_one_launch_from_many_slots(lens, budget, recent, weights):
    check_evict(lens, budget, recent, 64, 1, weights=KINDS[weights])


@pytest.mark.parametrize("lens, budget", [([300, 280], 272), ([9000, 8961], 8960), ([16417, 16390], 16384), ([20000, 16500], 64)])
def test_evict_in_one_launch_in_place(lens, budget):
    """Weights and positions in place, the lengths apart, which a loop gets by default."""
    rng = np.random.default_rng(budget)
    B, Hkv, page, recent = len(lens), 2, 64, 30
    cache, table = make_cache(lens, page, Hkv, rng)
    k, v = rows_of(rng, B, max(lens), Hkv, 12)
    adapld.kv8_append(cache, k.cuda(), v.cuda(), i32([0] * B), i32(lens))
    stride = max(lens) + 3
    w = np.floor(rng.random((B, Hkv, stride)) * 5000).astype(np.float32)
    p = np.stack([[rng.permutation(2 * stride)[:stride] for _ in range(Hkv)] for _ in range(B)]).astype(np.int32)
    want = arrays(cache)
    wo, po, lo = oracle.kv8_evict(w, p, lens, [2 * stride] * B, budget, recent, table, page, want)
    tw, tp = torch.from_numpy(w).cuda(), torch.from_numpy(p).cuda()
    gw, gp, gl = adapld.kv8_evict(cache, tw, tp, i32(lens), i32([2 * stride] * B), budget, recent, L_max=max(lens))
    assert gw is tw and gp is tp and gl.tolist() == lo
    for got, x in zip(arrays(cache), want):
        assert np.array_equal(got, x)
    for b in range(B):
        for g in range(Hkv):
            assert gw[b, g, :lo[b]].tolist() == [float(x) for x in wo[b * Hkv + g]] and gp[b, g, :lo[b]].tolist() == po[b * Hkv + g]
            assert np.array_equal(gw[b, g, lo[b]:].cpu().numpy(), w[b, g, lo[b]:])


# --------------------------------------------- the attention of a prompt's chunk

@pytest.mark.parametrize("Hq, T", [(32, 256), (64, 255), (4, 200)])
def test_verify_a_chunk_of_a_prompt(Hq, T):
    """Causal rows over a long cache: 2048, 4080 and 200 stacked rows a kv head."""
    check_heads(Case8([5003, 1500], Hq, 4, T, [T, T], 64, 5003, Hq, tree="chain"))
