"""The norm and rotation of prompts on the GPU against float64: more heads than a tree has,
several of them a wave, and above 196608 heads streamed.  Bounds as in
test_gpu_norm_rope.py.
"""
import math

import pytest
import torch

import paper_2606_05742_amd as adapld
from test_gpu_kv4 import i32

pytestmark = pytest.mark.gpu

# sequences, tokens, query and key heads; the number of heads is no multiple of those of a wave
SIZES = {"up to 196608": [(3, 403, 28, 4), (4, 1001, 5, 2)], "streamed": [(3, 2203, 28, 4), (4, 7100, 5, 2), (2, 6007, 17, 1)]}


def expected(x, weight, freqs, p, eps, interleaved):
    """The formula in float64, and the largest magnitude that takes part in each value."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * weight.double()
    h = freqs.numel()
    lo = slice(0, 2 * h, 2) if interleaved else slice(0, h)
    hi = slice(1, 2 * h, 2) if interleaved else slice(h, 2 * h)
    a = ((p[..., None] * freqs).double() * (2 * math.pi / 2.0 ** 64))[:, :, None]     # whole turns leave at 2^64
    out, size = y.clone(), y.abs()
    out[..., lo] = y[..., lo] * a.cos() - y[..., hi] * a.sin()
    out[..., hi] = y[..., hi] * a.cos() + y[..., lo] * a.sin()
    size[..., lo] = size[..., hi] = y[..., lo].abs() + y[..., hi].abs()
    return out, size


def check(q, k, freqs, base, offsets=None, counts=None, qw=None, kw=None, eps=1e-6, interleaved=False, into=None):
    """`into`: outputs to take; by default new ones, whose padding has to stay."""
    B, T = q.shape[:2]
    p = i32(base)[:, None].long() + (torch.arange(T, device="cuda") if offsets is None else offsets)
    live = torch.arange(T, device="cuda") < (torch.full((B, 1), T, device="cuda") if counts is None else i32(counts)[:, None])
    want = [expected(x, w, freqs, p, eps, interleaved) for x, w in ((q, qw), (k, kw))]
    qo, ko = into or (torch.full(x.shape, 77.0, dtype=torch.bfloat16, device="cuda") for x in (q, k))
    padding = [o[~live].clone() for o in (qo, ko)]
    adapld.qk_norm_rope(q, k, freqs, i32(base), offsets=offsets, counts=None if counts is None else i32(counts), q_weight=qw,
                        k_weight=kw, eps=eps, interleaved=interleaved, q_out=qo, k_out=ko)
    for o, (y, size), rest in zip((qo, ko), want, padding):
        assert ((o.double() - y).abs() <= 2.0 ** -8 * y.abs() + 2.0 ** -19 * size + 1e-38)[live].all()
        assert torch.equal(o[~live], rest)
    return qo, ko


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 32, 48, 64, 96, 128])
@pytest.mark.parametrize("sizes", sorted(SIZES))
def test_prompts(sizes, rot, interleaved):
    """Slices of a fused projection, every count of tokens, with and without the norm; then
    trees' offsets, every other token of a longer projection, without counts; then in place."""
    gen = torch.Generator(device="cuda").manual_seed(rot)
    freqs = adapld.rope_frequencies(rot, 10000.0)
    weight = lambda: (1 + 0.3 * torch.randn(128, generator=gen, device="cuda")).bfloat16()  # noqa: E731
    for B, T, Hq, Hkv in SIZES[sizes]:
        x = (torch.randn((B, T, Hq + 2 * Hkv, 128), generator=gen, device="cuda") * 2).bfloat16()
        q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv]
        base, qw, kw = [0, 131072, 2 ** 31 - 1, -9][:B], weight(), weight()
        check(q, k, freqs, base, counts=[T, T // 2 + 1, 0, T + 9][:B], qw=qw, kw=kw, interleaved=interleaved)
        check(q, k, freqs, base, counts=[T - 1, -3, T, 1][:B], kw=kw, eps=0.0, interleaved=interleaved)
        wide = (torch.randn((B, 2 * T, Hq + Hkv, 128), generator=gen, device="cuda")).bfloat16()
        offsets = torch.randint(-99, 9999, (B, T), generator=gen, device="cuda", dtype=torch.int32)
        check(wide[:, ::2, Hkv:], wide[:, 1::2, :Hkv], freqs, base, offsets=offsets, qw=qw, interleaved=interleaved)
        q, k = q.contiguous(), k.contiguous()
        check(q, k, freqs, base, counts=[T - 2, T, T, 5][:B], qw=qw, kw=kw, interleaved=interleaved, into=(q, k))
