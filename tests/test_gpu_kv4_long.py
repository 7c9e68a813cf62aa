"""The 4-bit cache's entry points at sizes near what they accept."""
import pytest
import torch

import paper_2606_05742_amd as adapld
from test_gpu_kv4 import i32

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
