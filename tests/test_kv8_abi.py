"""Refusals of the entry points around the 8-bit cache, on the host: every call
below carries an invalid argument or no sequence, which the library rejects (or
answers) before enqueueing anything."""
import ctypes
import os
import re

import pytest

from paper_2606_05742_amd import binding, build

OK, NULL, INVALID, UNSUPPORTED, WS_SMALL = 0, -1, -2, -3, -4
P = ctypes.c_void_p(0x10000)     # never dereferenced
ODD = ctypes.c_void_p(0x10008)   # 8-byte aligned only
N = None
MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def _args(names, **kw):
    assert set(kw) <= {n for n, _ in names}, kw
    return [kw.get(n, v) for n, v in names]


POOL = [("k_codes", P), ("k_scales", P), ("v_codes", P), ("v_scales", P)]
APPEND = [("k_new", P), ("v_new", P), ("rows", N), ("lens_old", P), ("lens_new", P), ("page_table", P), ("B", 2),
          ("n_src", 4), ("N", 4), ("Hkv", 2), ("D", 128), ("page_size", 16), ("n_pages", 20), ("max_pages", 8),
          *POOL, ("stream", N)]
VERIFY = [("q", P), *POOL, ("page_table", P), ("k_tree", P), ("v_tree", P), ("lens", P), ("node_count", P),
          ("tree_mask", P), ("B", 2), ("L_max", 100), ("T_max", 20), ("Hq", 8), ("Hkv", 2), ("D", 128),
          ("page_size", 16), ("n_pages", 20), ("max_pages", 8), ("scale", 0.1), ("out", P), ("lse", N), ("ws", P),
          ("ws_bytes", 1 << 30), ("stream", N)]
ROPE = [("q", P), ("k", P), ("q_batch", 4096), ("q_token", 1024), ("k_batch", 4096), ("k_token", 1024), ("q_weight", P),
        ("k_weight", P), ("freqs", P), ("base", P), ("offsets", N), ("counts", N), ("B", 2), ("T", 4), ("Hq", 8), ("Hkv", 2),
        ("D", 128), ("rot_dim", 64), ("interleaved", 0), ("eps", 1e-6), ("q_out", P), ("k_out", P), ("stream", N)]
WEIGHTS = [("q", P), ("lse", P), ("rows", N), ("k_codes", P), ("k_scales", P), ("page_table", P), ("lens_old", P),
           ("lens_new", P), ("first_position", P), ("B", 2), ("L_max", 100), ("T_max", 20), ("N", 20), ("Hq", 8),
           ("Hkv", 2), ("D", 128), ("page_size", 16), ("n_pages", 20), ("max_pages", 8), ("stride", 128), ("scale", 0.1),
           ("weights", P), ("weights_out", P), ("positions", P), ("stream", N)]
EVICT = [("weights", P), ("positions", P), ("lens", P), ("next_position", P), ("page_table", P), ("B", 2), ("L_max", 100),
         ("budget", 64), ("recent", 8), ("Hkv", 2), ("D", 128), ("page_size", 16), ("n_pages", 20), ("max_pages", 8),
         ("stride", 128), *POOL, ("weights_out", P), ("positions_out", P), ("lens_out", P), ("ws", P),
         ("ws_bytes", 1 << 30), ("stream", N)]
CALLS = {"adapld_qk_norm_rope": ROPE, "adapld_kv8_attn_weights": WEIGHTS, "adapld_kv8_evict": EVICT,
         "adapld_kv8_append": APPEND, "adapld_tree_verify_attn_kv8": VERIFY}
REQUIRED = {
    "adapld_qk_norm_rope": ["q", "k", "freqs", "base", "q_out", "k_out"],
    "adapld_kv8_attn_weights": ["q", "lse", "k_codes", "k_scales", "page_table", "lens_old", "lens_new",
                                "first_position", "weights", "weights_out", "positions"],
    "adapld_kv8_evict": ["weights", "positions", "lens", "next_position", "page_table", "k_codes", "k_scales",
                         "v_codes", "v_scales", "weights_out", "positions_out", "lens_out"],
    "adapld_kv8_append": ["k_new", "v_new", "lens_old", "lens_new", "page_table", "k_codes", "k_scales", "v_codes",
                          "v_scales"],
    "adapld_tree_verify_attn_kv8": ["q", "k_codes", "k_scales", "v_codes", "v_scales", "page_table", "k_tree",
                                    "v_tree", "tree_mask", "lens", "node_count", "out"]}
ALIGNED = {"adapld_kv8_attn_weights": ["q", "k_codes"], "adapld_kv8_evict": ["k_codes", "v_codes", "ws"],
           "adapld_qk_norm_rope": ["q", "k", "q_weight", "k_weight", "q_out", "k_out"],
           "adapld_kv8_append": ["k_new", "v_new", "k_codes", "v_codes"],
           "adapld_tree_verify_attn_kv8": ["q", "k_codes", "v_codes", "k_tree", "v_tree", "out"]}


def test_declared_and_exported(lib):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(build.INCLUDE, "adapld_kv8.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(adapld_\w+)\s*\(", src))
    assert names >= set(CALLS)
    for n in names:
        assert hasattr(lib, n) and n in binding.SIGNATURES


@pytest.mark.parametrize("call", sorted(CALLS))
def test_common_refusals(lib, call):
    f, names = getattr(lib, call), CALLS[call]
    has = {n for n, _ in names}
    assert f(*_args(names, B=0)) == OK
    assert f(*_args(names, B=-1)) == INVALID
    for p in REQUIRED[call]:
        assert f(*_args(names, **{p: N})) == NULL, p
    for p in ALIGNED[call]:
        assert f(*_args(names, **{p: ODD})) == INVALID, p
    if "n_pages" in has:
        for size in (0, 8, 15, 24, 48, 512, -16):
            assert f(*_args(names, page_size=size)) == INVALID, size
        assert f(*_args(names, n_pages=0)) == INVALID
        assert f(*_args(names, max_pages=0)) == INVALID
        assert f(*_args(names, n_pages=MAX // 16 + 1)) == UNSUPPORTED
        assert f(*_args(names, max_pages=MAX // 16 + 1)) == UNSUPPORTED
    assert f(*_args(names, D=64)) == UNSUPPORTED
    assert f(*_args(names, Hkv=0)) == INVALID


def test_append_refusals(lib):
    f = lib.adapld_kv8_append
    assert f(*_args(APPEND, n_src=3)) == INVALID            # without rows, tokens beyond the source
    assert f(*_args(APPEND, n_src=0, rows=P)) == INVALID
    assert f(*_args(APPEND, N=0)) == INVALID
    assert f(*_args(APPEND, B=1 << 14, N=1 << 16, n_src=1 << 16)) == UNSUPPORTED
    assert f(*_args(APPEND, N=MAX, n_src=MAX)) == UNSUPPORTED


def test_verify_refusals(lib):
    f = lib.adapld_tree_verify_attn_kv8
    for bad in (dict(L_max=0), dict(T_max=0), dict(Hq=0), dict(Hq=7), dict(L_max=129), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3.4e38)):
        assert f(*_args(VERIFY, **bad)) == INVALID, bad
    assert f(*_args(VERIFY, T_max=257)) == UNSUPPORTED
    assert f(*_args(VERIFY, L_max=(1 << 30) + 1, max_pages=(1 << 30) // 256 + 1, page_size=256)) == UNSUPPORTED
    need = lib.adapld_workspace_bytes(10, 2, 100, 0, 0, 20, 8, 2, 128)
    big = dict(L_max=2000, max_pages=200)
    need = lib.adapld_workspace_bytes(10, 2, 2000, 0, 0, 20, 8, 2, 128)
    assert need > 0
    assert f(*_args(VERIFY, ws_bytes=need - 1, **big)) == WS_SMALL
    assert f(*_args(VERIFY, ws=N, **big)) == NULL
    assert f(*_args(VERIFY, ws=ODD, **big)) == INVALID


def test_norm_rope_refusals(lib):
    f = lib.adapld_qk_norm_rope
    for bad in (dict(T=0), dict(Hq=0), dict(rot_dim=-16), dict(rot_dim=8), dict(rot_dim=144), dict(interleaved=2),
                dict(interleaved=-1), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(q_batch=-8),
                dict(q_token=1020), dict(k_batch=4), dict(k_token=-1024), dict(freqs=ctypes.c_void_p(0x10004))):
        assert f(*_args(ROPE, **bad)) == INVALID, bad
    assert f(*_args(ROPE, B=1 << 14, T=1 << 11)) == UNSUPPORTED
    assert f(*_args(ROPE, B=MAX, T=MAX, Hq=MAX, Hkv=MAX)) == UNSUPPORTED
    assert f(*_args(ROPE, B=1 << 13, T=1 << 13, Hq=1, Hkv=1)) == UNSUPPORTED   # a wave a token


def test_attn_weights_refusals(lib):
    f = lib.adapld_kv8_attn_weights
    for bad in (dict(L_max=0), dict(T_max=0), dict(N=0), dict(N=21), dict(Hq=0), dict(Hq=7), dict(L_max=129, stride=1000),
                dict(stride=99), dict(scale=0.0), dict(scale=float("nan")), dict(scale=3.4e38)):
        assert f(*_args(WEIGHTS, **bad)) == INVALID, bad
    assert f(*_args(WEIGHTS, T_max=257)) == UNSUPPORTED
    assert f(*_args(WEIGHTS, N=257, rows=P)) == UNSUPPORTED
    assert f(*_args(WEIGHTS, N=256, rows=P, Hq=1 << 20, Hkv=1)) == UNSUPPORTED
    assert f(*_args(WEIGHTS, T_max=256, N=1, Hq=1 << 20, Hkv=1)) == UNSUPPORTED
    assert f(*_args(WEIGHTS, B=1 << 22, L_max=16)) == UNSUPPORTED                # a workgroup a kv head
    assert f(*_args(WEIGHTS, B=1 << 16, Hkv=8, L_max=1 << 13, max_pages=1 << 9, stride=1 << 13)) == UNSUPPORTED


def test_evict_refusals(lib):
    f, need = lib.adapld_kv8_evict, lib.adapld_kv8_evict_workspace_bytes
    for bad in (dict(L_max=0), dict(L_max=129, stride=1000), dict(stride=99), dict(budget=0), dict(budget=-16), dict(budget=24),
                dict(recent=-1)):
        assert f(*_args(EVICT, **bad)) == INVALID, bad
    assert need(2, 2, 100, 64) == 4 * (64 + 36 + 1) * 4 and need(2, 2, 64, 64) == 0 and need(0, 2, 100, 64) == 0
    assert f(*_args(EVICT, ws_bytes=need(2, 2, 100, 64) - 1)) == WS_SMALL
    assert f(*_args(EVICT, ws=N)) == NULL
    assert f(*_args(EVICT, B=1 << 22, Hkv=1)) == UNSUPPORTED
    assert f(*_args(EVICT, B=1 << 16, Hkv=8, L_max=4096, budget=2048, max_pages=256, stride=4096)) == UNSUPPORTED
