"""What the header promises of dkv_paged_query_attn at its edges: lists that name slots outside their pages."""

import numpy as np
import pytest
import torch

from test_gpu_paged_query import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


@pytest.mark.parametrize("R", [32, 64, 256, 1024])
@pytest.mark.parametrize("new", [[6, 9], [80, 140]])
def test_entries_whose_slots_end_below_zero(d, new, R):
    """An end far below zero, where end - slot passes the smallest int32 for the later runs of the page, names no slot;
    nor do a first slot and an end at the largest int32."""
    rng = np.random.default_rng([R, new[0]])
    x = Batch(rng, [8 * R, 7 * R], new, 2, 4, 64, R)
    least, most = -2 ** 31, 2 ** 31 - 1
    for s in range(4):
        x.entries[s, 1, 2:] = (0, least)
        x.entries[s, 2, 2:] = (0, least + 31)
        x.entries[s, 3, 2:] = (0, least + R - 32)
        x.entries[s, 4, 2:] = (0, most)
        x.entries[s, 5, 2:] = (most, most)
    x.check(d)
