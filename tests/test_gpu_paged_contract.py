"""What the header promises of dkv_paged_query_attn at its edges: lists that name slots outside their pages; equal
bits on every call."""

import numpy as np
import pytest
import torch

from test_gpu_paged_query import Batch
from test_paged_plan_cpu import BATCHES, deal, unit_costs

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


@pytest.mark.parametrize("batch", BATCHES)
def test_the_form_of_a_call_does_not_depend_on_timing(d, batch):
    """Whether query tiles stay whole is what the host's model of the plan says, call after call, and so are the bits.
    Every page of the long contexts is one of 300."""
    held, new = batch
    Hkv, G, dim, R, pool, B = 8, 4, 128, 128, 300, len(held)
    gen = torch.Generator(device="cuda").manual_seed(B)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    i32 = lambda x: torch.as_tensor(np.asarray(x), device="cuda").to(torch.int32)  # noqa: E731
    tokens, most = sum(new), max(new)
    grown = [h + n for h, n in zip(held, new)]
    count = [-(-n // R) for n in grown]
    entries = torch.zeros((B * Hkv, max(count), 4), dtype=torch.int32, device="cuda")
    entries[..., 0] = torch.randint(pool, entries.shape[:2], generator=gen, device="cuda")
    entries[..., 1] = torch.arange(max(count), device="cuda")
    end = i32(grown).repeat_interleave(Hkv)[:, None] - entries[..., 1] * R
    entries[..., 3] = end.clamp(0, R)
    hint = sum(count) * R * Hkv
    ws = torch.zeros(d.dkv_paged_query_workspace_bytes(B, Hkv * G, Hkv, dim, tokens, most, hint), dtype=torch.uint8,
                     device="cuda")
    args = (rand(tokens, Hkv * G, dim), i32(np.concatenate([[0], np.cumsum(new)])), i32(held), rand(pool, R, dim),
            rand(pool, R, dim), entries, i32(np.repeat(count, Hkv)), 1.0 / np.sqrt(dim))
    outs = [torch.empty((tokens, Hkv * G, dim), device="cuda") for _ in range(2)]
    whole = deal(unit_costs(held, new, Hkv, G), own_length=False)
    for i in range(30):
        d.dkv_paged_query_attn(*args, outs[min(i, 1)], ws, Hkv, most, rows_hint=hint)
        assert int(ws[8:12].view(torch.int32)) == int(whole), i  # the plan's third word
        assert torch.equal(outs[0], outs[min(i, 1)]), i
