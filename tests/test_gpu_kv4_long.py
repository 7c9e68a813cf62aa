"""The 4-bit cache's entry points at sizes near what they accept."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_05742_amd as adapld
from test_gpu_kv4 import DELTA, bf16, f64, i32

pytestmark = pytest.mark.gpu

INT_MAX = 2 ** 31 - 1


@pytest.mark.parametrize("in_place", (True, False))
def test_the_longest_slot_map(in_place):
    """As many slots of one sequence as the entry point takes: by a launch of
    their own (the count in place) and beside the pages."""
    cache = adapld.Kv4Cache.allocate(64, 16, 1, 1, 64)
    lens_new = 1000
    slots = torch.full((1, INT_MAX), -7, dtype=torch.int32, device="cuda")
    count = cache.free_count if in_place else i32([0])
    _, granted = adapld.page_map(cache, i32([0]), i32([lens_new]), slot_map=slots, free_count_out=count)
    assert granted.tolist() == [1] and count.tolist() == [1]
    # pages 0, 1, .. are handed out from the top of the stack, in order
    assert torch.equal(slots[0, :lens_new], torch.arange(lens_new, dtype=torch.int32, device="cuda"))
    assert bool((slots[0, lens_new:] == -1).all())


def test_bytes_beyond_32_bits():
    """Rows of pages whose byte offsets pass 32 bits, against bytes and values of
    the reference: offsets cut to 32 bits alike in every kernel would meet in
    the pages 4 GiB before, which stay as they were."""
    page, Hkv, Hq, L = 256, 8, 16, 700
    n_pages = (5 << 30) // (page * Hkv * 64)
    alias = (1 << 32) // (page * Hkv * 64)
    cache = adapld.Kv4Cache.allocate(n_pages, page, Hkv, 1, 3)
    arrays = (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)
    table = [n_pages - 1, 1, n_pages - 2]
    cache.page_table.copy_(i32([table]))
    far, near = (n_pages - 1, n_pages - 2), (n_pages - 1 - alias, n_pages - 2 - alias)
    assert not set(near) & set(table) and min(near) > 0
    for t in arrays:
        for p in far + near:
            t[p] = 0x65
    rng = np.random.default_rng(31)
    k, v = (bf16(rng.standard_normal((1, L, Hkv, 128))) for _ in range(2))
    pos = np.arange(L)
    slots = i32((np.array(table)[pos // page] * page + pos % page)[None].tolist())
    adapld.kv4_append(cache, k.cuda(), v.cuda(), slots)
    values = []
    for x, codes, scales in ((k, arrays[0], arrays[1]), (v, arrays[2], arrays[3])):
        code, e = oracle.kv4_quantise(f64(x[0]))                  # [L, Hkv, ..]
        packed = oracle.kv4_pack(code)
        values.append(oracle.kv4_values(packed, e))
        for got, want in ((codes, packed), (scales, e)):
            for i, p in enumerate(table):
                w = want[i * page:(i + 1) * page].transpose(1, 0, 2)   # [Hkv, rows, bytes]
                g = got[p].cpu().numpy()
                assert np.array_equal(g[:, :w.shape[1]], w), p
                assert p not in far or (g[:, w.shape[1]:] == 0x65).all(), p
            for p in near:
                assert bool((got[p] == 0x65).all()), p
    for got, want in zip(adapld.kv4_gather(cache, slots), values):
        assert np.array_equal(f64(got[0]), want)
    kq, vq = (np.ascontiguousarray(x.transpose(1, 0, 2))[None] for x in values)
    for T in (1, 40):                                              # either kernel of the attention
        q = bf16(rng.standard_normal((1, T, Hq, 128))).cuda()
        out, lse = adapld.tree_verify_attn_kv4(q, cache, i32([L]), i32([T]), L_max=L)
        o, l, spread, _ = oracle.kv4_verify(f64(q), kq, vq, [L], [T])
        assert (np.abs(f64(out) - o) <= 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2 * DELTA) * spread).all()
        assert np.abs(f64(lse) - l).max() <= 1e-4
