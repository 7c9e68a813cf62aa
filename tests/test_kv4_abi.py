"""Refusals of the 4-bit cache's entry points and the bounds of its layout, on
the host: every call below carries an invalid argument or no sequence, which
the library rejects (or answers) before enqueueing anything."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2606_05742_amd as adapld
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


MAP = [("lens_old", P), ("lens_new", P), ("B", 2), ("page_size", 16), ("max_pages", 8), ("n_pages", 20), ("N", 4),
       ("page_table", P), ("free_pages", P), ("free_count", P), ("free_count_out", P), ("slot_map", P),
       ("granted", P), ("stream", N)]
APPEND = [("k_new", P), ("v_new", P), ("rows", N), ("slot_map", P), ("B", 2), ("n_src", 4), ("N", 4), ("Hkv", 2),
          ("D", 128), ("page_size", 16), ("n_pages", 20), ("k_codes", P), ("k_scales", P), ("v_codes", P),
          ("v_scales", P), ("stream", N)]
GATHER = [("k_codes", P), ("k_scales", P), ("v_codes", P), ("v_scales", P), ("slot_map", P), ("B", 2), ("N", 4),
          ("Hkv", 2), ("D", 128), ("page_size", 16), ("n_pages", 20), ("k_out", P), ("v_out", P), ("stream", N)]
VERIFY = [("q", P), ("k_codes", P), ("k_scales", P), ("v_codes", P), ("v_scales", P), ("page_table", P),
          ("k_tree", P), ("v_tree", P), ("lens", P), ("node_count", P), ("tree_mask", P), ("B", 2), ("L_max", 100),
          ("T_max", 20), ("Hq", 8), ("Hkv", 2), ("D", 128), ("page_size", 16), ("n_pages", 20), ("max_pages", 8),
          ("scale", 0.1), ("out", P), ("lse", N), ("ws", P), ("ws_bytes", 1 << 30), ("stream", N)]
CALLS = {"adapld_kv4_page_map": MAP, "adapld_kv4_append": APPEND, "adapld_kv4_gather": GATHER,
         "adapld_tree_verify_attn_kv4": VERIFY}
REQUIRED = {
    "adapld_kv4_page_map": ["lens_old", "lens_new", "page_table", "free_pages", "free_count", "free_count_out",
                            "slot_map", "granted"],
    "adapld_kv4_append": ["k_new", "v_new", "slot_map", "k_codes", "k_scales", "v_codes", "v_scales"],
    "adapld_kv4_gather": ["k_out", "v_out", "slot_map", "k_codes", "k_scales", "v_codes", "v_scales"],
    "adapld_tree_verify_attn_kv4": ["q", "k_codes", "k_scales", "v_codes", "v_scales", "page_table", "k_tree",
                                    "v_tree", "tree_mask", "lens", "node_count", "out"]}


def test_declared_and_exported(lib):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(build.INCLUDE, "adapld.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(adapld_\w*kv4\w*)\s*\(", src))
    assert names == set(CALLS)
    for n in names:
        assert hasattr(lib, n) and n in binding.SIGNATURES


@pytest.mark.parametrize("call", sorted(CALLS))
def test_common_refusals(lib, call):
    f, names = getattr(lib, call), CALLS[call]
    assert f(*_args(names, B=0)) == OK
    assert f(*_args(names, B=-1)) == INVALID
    for p in REQUIRED[call]:
        assert f(*_args(names, **{p: N})) == NULL, p
    for size in (0, 8, 15, 24, 48, 512, -16):
        assert f(*_args(names, page_size=size)) == INVALID, size
    assert f(*_args(names, n_pages=0)) == INVALID
    assert f(*_args(names, n_pages=MAX // 16 + 1)) == UNSUPPORTED
    assert f(*_args(names, n_pages=MAX, page_size=256)) == UNSUPPORTED
    if any(n == "D" for n, _ in names):
        assert f(*_args(names, D=64)) == UNSUPPORTED
        assert f(*_args(names, k_codes=ODD)) == INVALID
        assert f(*_args(names, v_codes=ODD)) == INVALID
        assert f(*_args(names, k_scales=ctypes.c_void_p(0x10002))) == INVALID
        assert f(*_args(names, v_scales=ctypes.c_void_p(0x10001))) == INVALID
        assert f(*_args(names, Hkv=0)) == INVALID


def test_page_map_refusals(lib):
    f = lib.adapld_kv4_page_map
    assert f(*_args(MAP, N=-1)) == INVALID
    assert f(*_args(MAP, max_pages=0)) == INVALID
    assert f(*_args(MAP, max_pages=MAX // 16 + 1)) == UNSUPPORTED
    assert f(*_args(MAP, B=65536)) == UNSUPPORTED
    assert f(*_args(MAP, B=60000, max_pages=40000)) == UNSUPPORTED
    assert f(*_args(MAP, B=60000, N=40000)) == UNSUPPORTED
    assert f(*_args(MAP, N=0, slot_map=N, B=0)) == OK


def test_row_refusals(lib):
    f, g = lib.adapld_kv4_append, lib.adapld_kv4_gather
    assert f(*_args(APPEND, n_src=3)) == INVALID            # without rows, slots beyond the source
    assert f(*_args(APPEND, n_src=0, rows=P)) == INVALID
    assert f(*_args(APPEND, N=0)) == INVALID
    assert f(*_args(APPEND, k_new=ODD)) == INVALID
    assert f(*_args(APPEND, v_new=ODD)) == INVALID
    assert f(*_args(APPEND, B=1 << 14, N=1 << 13, n_src=1 << 13)) == UNSUPPORTED
    assert g(*_args(GATHER, k_out=ODD)) == INVALID
    assert g(*_args(GATHER, v_out=ODD)) == INVALID
    assert g(*_args(GATHER, N=0)) == INVALID
    assert g(*_args(GATHER, B=1 << 14, N=1 << 13)) == UNSUPPORTED


def test_verify_refusals(lib):
    f = lib.adapld_tree_verify_attn_kv4
    ok = dict(k_tree=N, v_tree=N, tree_mask=N)
    assert f(*_args(VERIFY, B=0, **ok)) == OK
    for some in (dict(k_tree=N), dict(k_tree=N, v_tree=N), dict(v_tree=N, tree_mask=N)):
        assert f(*_args(VERIFY, **some)) == NULL
    assert f(*_args(VERIFY, L_max=0)) == INVALID
    assert f(*_args(VERIFY, L_max=129)) == INVALID           # beyond 8 pages of 16
    assert f(*_args(VERIFY, T_max=0)) == INVALID
    assert f(*_args(VERIFY, T_max=257)) == UNSUPPORTED
    assert f(*_args(VERIFY, Hq=7)) == INVALID
    assert f(*_args(VERIFY, Hq=0)) == INVALID
    assert f(*_args(VERIFY, max_pages=0)) == INVALID
    assert f(*_args(VERIFY, max_pages=MAX // 16 + 1)) == UNSUPPORTED
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert f(*_args(VERIFY, scale=scale)) == INVALID
    for p in ("q", "out", "k_tree", "v_tree"):
        assert f(*_args(VERIFY, **{p: ODD})) == INVALID, p
    assert f(*_args(VERIFY, B=1 << 20, Hkv=8)) == UNSUPPORTED
    big = dict(B=1, L_max=16 * 1024, max_pages=1024)
    need = lib.adapld_workspace_bytes(8, 1, 16 * 1024, 0, 0, 20, 8, 2, 128)
    assert need > 0
    assert f(*_args(VERIFY, ws_bytes=need - 1, **big)) == WS_SMALL
    assert f(*_args(VERIFY, ws=N, **big)) == NULL
    assert f(*_args(VERIFY, ws=ODD, **big)) == INVALID


def test_scale_refusals(lib):
    """A finite scale that no longer fits fp32 in units of log2."""
    for scale in (3.4e38, 2.4e38):
        assert lib.adapld_tree_verify_attn_kv4(*_args(VERIFY, scale=scale)) == INVALID


def test_workspace_sizes(lib):
    ws = lib.adapld_workspace_bytes
    for bad in (dict(T_max=0), dict(T_max=257), dict(Hq=7), dict(Hkv=0), dict(B=0), dict(L=0), dict(L=(1 << 30) + 1)):
        a = dict(B=2, L=4096, T_max=20, Hq=8, Hkv=2, **{}) | bad
        assert ws(8, a["B"], a["L"], 0, 0, a["T_max"], a["Hq"], a["Hkv"], 128) == 0, bad
    # every split is within what one workgroup holds, up to the largest length
    for L in (1, 64, 65, 40000, 1 << 20, 1 << 30):
        assert ws(8, 1, L, 0, 0, 1, 8, 8, 128) >= (0 if L <= 32768 else 8 * (L // 32768) * 520)


def test_binding_refuses_host_tensors_and_shapes():
    cache = adapld.Kv4Cache.allocate(4, 16, 2, 1, 2, device="cpu")
    assert cache.n_pages == 4 and cache.Hkv == 2 and cache.free_pages.tolist() == [3, 2, 1, 0]
    lens = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(adapld.AdapldError):
        adapld.page_map(cache, lens, lens, 1)
    k = torch.zeros((1, 1, 2, 128), dtype=torch.bfloat16)
    slots = torch.zeros((1, 1), dtype=torch.int32)
    with pytest.raises(adapld.AdapldError):
        adapld.kv4_append(cache, k, k, slots)
    with pytest.raises(adapld.AdapldError):
        adapld.kv4_append(cache, k[:, :, :1], k[:, :, :1], slots)      # kv heads
    with pytest.raises(adapld.AdapldError):
        adapld.kv4_gather(cache, slots)
    with pytest.raises(adapld.AdapldError):
        adapld.tree_verify_attn_kv4(torch.zeros((1, 1, 4, 128), dtype=torch.bfloat16), cache, lens, lens)


LAYOUT = r"""
#include <hip/hip_runtime.h>
#include <climits>
#include <cstdio>
#include "kv4.h"
using namespace adapld;
int main() {
  const int ids[] = {INT_MIN, -1, 0, 1, 6, 7, 8, INT_MAX};
  for (int shift = 4; shift <= 8; ++shift) {
    if (log2_pow2(1 << shift) != shift) return 1;
    for (int n_pages : {1, 2, 7}) for (int Hkv : {1, 3, 8}) {
      const size_t rows = ((size_t)n_pages * Hkv) << shift;
      for (int id : ids) {
        const int p = kv4_page_in_pool(id, n_pages);
        if (p < 0 || p >= n_pages || (id >= 0 && id < n_pages && p != id)) return 2;
        for (int g = 0; g < Hkv; ++g) for (int off : {0, (1 << shift) - 1})
          if (kv4_row(p, g, off, Hkv, shift) >= rows) return 3;
      }
    }
    // the last row of the largest pool, beyond 32 bits
    const int n = INT_MAX >> shift;
    if (kv4_row(n - 1, 63, (1 << shift) - 1, 64, shift) + 1 != ((size_t)n * 64) << shift) return 4;
  }
  puts("ok");
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_layout_stays_in_the_pool(tmp_path):
    """Rows of any page id, clamped as the attention clamps it, lie in the pool."""
    src, exe = tmp_path / "layout.cpp", tmp_path / "layout"
    src.write_text(LAYOUT)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(build.hipcc())))
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-I",
                    build.INCLUDE, "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.returncode


@pytest.mark.skipif(shutil.which("g++") is None or "ADAPLD_LIB" in os.environ, reason="needs g++; not from its own child")
def test_refusals_under_sanitizers():
    """This file's calls against the C-ABI glue under AddressSanitizer and UBSan."""
    import sys
    lib = build.build_host_sanitized()
    env = dict(os.environ, ADAPLD_LIB=lib, LD_PRELOAD=build.sanitizer_preload(),
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "-k", "refusals or workspace",
                        os.path.abspath(__file__)], cwd=build.ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
