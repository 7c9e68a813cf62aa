"""The 8-bit cache's larger calls on the GPU: prompts whose rows are streamed into it.
Stored bytes are exact.
"""
import math

import numpy as np
import pytest

from test_gpu_kv8 import check_append, rows_of

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
