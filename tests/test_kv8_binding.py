"""What the binding of the operators around the 8-bit cache hands to the library,
and what it refuses itself, on the host: the library is replaced by one that notes
its calls, and host tensors pass for those of the current device."""
import math

import pytest
import torch

import paper_2606_05742_amd as adapld
from paper_2606_05742_amd import AdapldError
from test_kv4_binding import bf16, i32, lib  # noqa: F401


def cache_of(bits=8, n_pages=4, page_size=32, Hkv=2, B=1, max_pages=3):
    return (adapld.Kv8Cache if bits == 8 else adapld.Kv4Cache).allocate(n_pages, page_size, Hkv, B, max_pages, device="cpu")


def test_caches_of_the_other_width_are_refused(lib):  # noqa: F811
    q, kv, n = bf16(1, 2, 4, 128), bf16(1, 3, 2, 128), i32([1])
    four, eight, w = cache_of(4), cache_of(8), torch.zeros((1, 2, 96))
    for call in (lambda: adapld.kv8_append(four, kv, kv, n, n), lambda: adapld.tree_verify_attn_kv8(q, four, n, n),
                 lambda: adapld.kv4_append(eight, kv, kv, i32([[0, 1, 2]])), lambda: adapld.kv4_gather(eight, i32([[0]])),
                 lambda: adapld.tree_verify_attn_kv4(q, eight, n, n),
                 lambda: adapld.kv8_attn_weights(four, q, w, n, n, n, w, i32([[[0]]])),
                 lambda: adapld.kv8_evict(four, w, i32([[[0]]]), n, n, 16)):
        with pytest.raises(AdapldError, match="bits a value"):
            call()
    assert not lib.calls


def test_append_passes_the_sizes(lib):  # noqa: F811
    c = cache_of()
    adapld.kv8_append(c, bf16(1, 3, 2, 128), bf16(1, 3, 2, 128), i32([4]), i32([6]))
    adapld.kv8_append(c, bf16(1, 3, 2, 128), bf16(1, 3, 2, 128), i32([4]), i32([6]), rows=i32([[2, 0, 1, 1]]))
    adapld.kv8_append(c, bf16(1, 3, 2, 128), bf16(1, 3, 2, 128), i32([4]), i32([6]), N=2)
    assert [a[6:14] for name, a in lib.calls] == [(1, 3, n, 2, 128, 32, 4, 3) for n in (3, 4, 2)]
    for bad in (bf16(1, 3, 1, 128), bf16(2, 3, 2, 128), bf16(1, 3, 2, 64)):
        with pytest.raises(AdapldError):
            adapld.kv8_append(c, bad, bad, i32([4]), i32([6]))
    with pytest.raises(AdapldError):
        adapld.kv8_append(c, bf16(1, 3, 2, 128), bf16(1, 3, 2, 128), i32([4]), i32([6]), rows=i32([[2, 0]]), N=3)
    with pytest.raises(AdapldError):
        adapld.kv8_append(c, bf16(1, 3, 2, 128), bf16(1, 3, 2, 128), i32([4, 5]), i32([6]))


def test_scales_of_another_shape_are_refused(lib):  # noqa: F811
    c = cache_of()
    c.k_scales = torch.zeros((4, 2, 4), dtype=torch.uint8)
    with pytest.raises(AdapldError, match="k_scales"):
        adapld.kv8_append(c, bf16(1, 3, 2, 128), bf16(1, 3, 2, 128), i32([4]), i32([6]))
    assert not lib.calls


def test_norm_rope_strides(lib):  # noqa: F811
    x = bf16(2, 5, 6 * 128)
    q, k = x[..., :512].unflatten(-1, (4, 128)), x[..., 512:640].unflatten(-1, (1, 128))
    f = adapld.rope_frequencies(64, device="cpu")
    adapld.qk_norm_rope(q, k, f, i32([0, 1]))
    adapld.qk_norm_rope(q[:, ::2], k[:, ::2], f, i32([0, 1]))
    assert [a[2:6] for _, a in lib.calls] == [(5 * 768, 768, 5 * 768, 768), (5 * 768, 2 * 768, 5 * 768, 2 * 768)]
    assert lib.calls[0][1][12:19] == (2, 5, 4, 1, 128, 64, 0)
    one = torch.empty_strided((1, 1, 4, 128), (3, 5, 128, 1), dtype=torch.bfloat16)
    adapld.qk_norm_rope(one, one[:, :, :1], f, i32([0]))
    assert lib.calls.pop()[1][2:6] == (0, 0, 0, 0)          # strides of single entries mean nothing
    for bad in (dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(k=bf16(2, 4, 1, 128)), dict(q=q.float()),
                dict(freqs=f.int()), dict(q_weight=bf16(64)), dict(offsets=i32([[0, 1]])), dict(base=i32([1]))):
        with pytest.raises(AdapldError):
            adapld.qk_norm_rope(**(dict(q=q, k=k, freqs=f, base=i32([0, 1])) | bad))
    assert len(lib.calls) == 2


def test_frequencies():
    f = adapld.rope_frequencies(4, rad_per_token=[2 * math.pi * 0.25, -2 * math.pi * 0.25], device="cpu")
    assert f.tolist() == [1 << 62, -(1 << 62)]
    assert adapld.rope_frequencies(2, rad_per_token=[2 * math.pi * 0.5], device="cpu").tolist() == [-(1 << 63)]
    assert adapld.rope_frequencies(0, device="cpu").tolist() == []
    for bad in (dict(rot_dim=3), dict(rot_dim=-2), dict(rot_dim=4, rad_per_token=[1.0]),
                dict(rot_dim=2, rad_per_token=[math.inf])):
        with pytest.raises(AdapldError):
            adapld.rope_frequencies(**bad, device="cpu")


def test_weights_and_eviction_pass_the_sizes(lib):  # noqa: F811
    c, n = cache_of(), i32([4])
    w, p = torch.zeros((1, 2, 80)), torch.zeros((1, 2, 80), dtype=torch.int32)
    q, lse = bf16(1, 5, 4, 128), torch.zeros((1, 4, 5))
    assert adapld.kv8_attn_weights(c, q, lse, n, n, n, w, p)[0] is w
    adapld.kv8_attn_weights(c, q, lse, n, n, n, w, p, rows=i32([[1, 2]]), L_max=70, weights_out=w.clone())
    assert [a[9:20] for _, a in lib.calls] == [(1, 80, 5, 5, 4, 2, 128, 32, 4, 3, 80), (1, 70, 5, 2, 4, 2, 128, 32, 4, 3, 80)]
    lib.calls.clear()
    wo, po, lo = adapld.kv8_evict(c, w, p, n, n, 32, 7, ws=torch.zeros(4096, dtype=torch.uint8))
    assert wo is w and po is p and lo.shape == (1,)
    assert lib.calls[0][1][5:15] == (1, 80, 32, 7, 2, 128, 32, 4, 3, 80)
    ws = torch.zeros(4096, dtype=torch.uint8)
    for bad in (dict(weights=w[:, :1]), dict(weights=w.double()), dict(positions=p[..., :79]), dict(lens=i32([1, 2])),
                dict(positions_out=p[..., :79])):
        with pytest.raises(AdapldError):
            adapld.kv8_evict(**(dict(cache=c, weights=w, positions=p, lens=n, next_position=n, budget=32, ws=ws) | bad))
    for bad in (dict(q=bf16(1, 5, 4, 64)), dict(lse=lse[..., :4]), dict(weights=w[0]), dict(rows=i32([[1]]), N=2),
                dict(positions=p.long())):
        with pytest.raises(AdapldError):
            adapld.kv8_attn_weights(**(dict(cache=c, q=q, lse=lse, lens_old=n, lens_new=n, first_position=n, weights=w,
                                            positions=p) | bad))
    assert len(lib.calls) == 1
