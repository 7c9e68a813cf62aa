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


def _calls(c):
    """One call of each kind on a cache of two sequences and two kv heads."""
    lens, slots, x = i32([3, 3]), i32([[0], [1]]), bf16(2, 1, 2, 128)
    return {
        "page_map": lambda: adapld.page_map(c, lens, lens, slot_map=slots, granted=i32([0, 0])),
        "append": lambda: adapld.kv4_append(c, x, x, slots),
        "gather": lambda: adapld.kv4_gather(c, slots, k_out=x, v_out=x),
        "verify": lambda: adapld.tree_verify_attn_kv4(
            bf16(2, 1, 4, 128), c, lens, lens, L_max=16, out=bf16(2, 1, 4, 128), lse=torch.zeros((2, 4, 1)),
            ws=torch.zeros(16, dtype=torch.uint8))}


POOL = ("append", "gather", "verify")
# What may become of a buffer at its old address: another shape, fewer pages,
# other strides, another type.
SAME_ADDRESS = {
    "half": lambda t: t[:t.shape[0] // 2],
    "flat": lambda t: t.view(-1),
    "transposed": lambda t: t.transpose(0, -1),
    "strided": lambda t: t[::2],
    "int8": lambda t: t.view(torch.int8)}


@pytest.mark.parametrize("name, kinds, hows", [
    *((name, POOL, sorted(SAME_ADDRESS)) for name in ("k_codes", "k_scales", "v_codes", "v_scales")),
    ("page_table", ("page_map", "verify"), ("half", "flat", "transposed", "int8")),
    ("free_pages", ("page_map",), ("strided", "int8")), ("free_count", ("page_map",), ("half", "int8"))])
def test_buffers_reshaped_at_the_same_address(lib, name, kinds, hows):
    """A buffer that no longer fits is refused though its address is the old
    one, and every call goes on once it fits again."""
    c = cache_of(B=2)
    calls = _calls(c)
    for kind in kinds:
        calls[kind]()
    t = getattr(c, name)
    whole = t.data
    for how in hows:
        lib.calls.clear()
        t.data = SAME_ADDRESS[how](whole)
        assert t.numel() == 0 or t.data_ptr() == whole.data_ptr()
        for kind in kinds:
            for _ in range(2):
                with pytest.raises(adapld.AdapldError):
                    calls[kind]()
        assert lib.calls == [], how
        t.data = whole
        for kind in kinds:
            calls[kind]()
        assert len(lib.calls) == len(kinds)


def test_smaller_pool_at_the_same_address(lib):
    """Buffers that shrink together are the smaller cache from the next call on."""
    c = cache_of(B=2, max_pages=2)
    calls = _calls(c)
    for kind in POOL:
        calls[kind]()
    lib.calls.clear()
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        t = getattr(c, name)
        t.data = t.data[:3]
    c.page_table.data = c.page_table.data[:, :1].contiguous()
    for kind in POOL:
        calls[kind]()
    sizes = {name: args for name, args in lib.calls}
    assert sizes["adapld_kv4_append"][10] == 3 and sizes["adapld_kv4_gather"][10] == 3
    assert sizes["adapld_tree_verify_attn_kv4"][18:20] == (3, 1)     # n_pages, max_pages


@pytest.mark.parametrize("n", (3, 5))
def test_page_map_refuses_a_stack_of_another_pool(lib, n):
    """Page ids of a longer stack lie outside the pool: their rows would be
    dropped by the append and read as another page's by the attention; a shorter
    one takes ids of the pool for pages outside."""
    c = cache_of(B=2)
    call = _calls(c)["page_map"]
    call()
    whole = c.free_pages
    c.free_pages = torch.zeros(n, dtype=torch.int32)
    for _ in range(2):
        with pytest.raises(adapld.AdapldError):
            call()
    c.free_pages = whole
    call()
    whole.data = whole.data[:3]                 # in place
    with pytest.raises(adapld.AdapldError):
        call()
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        setattr(c, name, getattr(c, name)[:3])
    call()                                      # the pool of the smaller stack
    c.k_codes.data = c.k_codes.data[:2]
    with pytest.raises(adapld.AdapldError):
        call()
    c.k_codes = None                            # a stack without a pool
    call()
    assert [args[5] for _, args in lib.calls] == [4, 4, 3, 3]
