"""What the binding of the 4-bit cache hands to the library, on the host: the
library is replaced by one that notes its calls, and host tensors pass for
those of the current device."""
import pytest
import torch

import paper_2606_05742_amd as adapld
from paper_2606_05742_amd import binding


class Library:
    """Notes (name, arguments) of every call and answers ADAPLD_OK."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    noted = Library()
    monkeypatch.setattr(binding, "load_library", lambda *a: noted)
    monkeypatch.setattr(binding, "_device_of", lambda t, name: -1)   # a host tensor's device index
    monkeypatch.setattr(binding, "_stream_on", lambda stream, dev: None)
    return noted


def i32(x):
    return torch.tensor(x, dtype=torch.int32)


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def cache_of(n_pages=4, page_size=16, Hkv=2, B=1, max_pages=3):
    return adapld.Kv4Cache.allocate(n_pages, page_size, Hkv, B, max_pages, device="cpu")


def narrow_cache():
    """A cache of 64 dimensions, from the caller's own buffers."""
    u8 = lambda n: torch.zeros((4, 2, 16, n), dtype=torch.uint8)  # noqa: E731
    return adapld.Kv4Cache(k_codes=u8(32), k_scales=u8(2), v_codes=u8(32), v_scales=u8(2), page_table=i32([[0, 1]]),
                           free_pages=i32([3, 2, 1, 0]), free_count=i32([4]), page_size=16)


def test_append_passes_the_sizes(lib):
    c = cache_of()
    adapld.kv4_append(c, bf16(1, 3, 2, 128), bf16(1, 3, 2, 128), i32([[0, 1, -1]]))
    (name, args), = lib.calls
    assert name == "adapld_kv4_append" and args[4:11] == (1, 3, 3, 2, 128, 16, 4)


def test_append_refuses_rows_wider_than_the_cache(lib):
    """Rows of 128 dimensions do not fit the code rows of a cache of 64."""
    slots = i32([[0]])
    with pytest.raises(adapld.AdapldError):
        adapld.kv4_append(narrow_cache(), bf16(1, 1, 2, 128), bf16(1, 1, 2, 128), slots)
    with pytest.raises(adapld.AdapldError):
        adapld.kv4_append(cache_of(), bf16(1, 1, 2, 64), bf16(1, 1, 2, 64), slots)
    assert lib.calls == []


def test_allocate_refuses_other_head_dimensions():
    for D in (64, 96, 256, 0):
        with pytest.raises(adapld.AdapldError):
            adapld.Kv4Cache.allocate(4, 16, 2, 1, 2, D=D, device="cpu")
