"""Compressed requests beside others in one batch: dkv_page_extend writes every list in the format of an unpruned
cache, and dkv_page_select then lists the compressed requests' segments again, from the mask of their selection and the
pages that they have by then."""

import numpy as np
import pytest
import torch

from _helpers import row_rel_err
from test_gpu_paged_query import DEV, _bf16, _dev
from test_paged_precision_cpu import LIMIT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


@pytest.mark.parametrize("R,dim", [(32, 64), (64, 128), (256, 128)])
def test_compressed_requests_grow_beside_others(d, R, dim):
    """Prompts, a selection of two of the three, their unused pages to the stack and (through it) to the third; then
    chunks and single tokens of all, past several page ends, each step checked against dense attention."""
    rng = np.random.default_rng([R, dim])
    B, Hkv, G, T = 3, 2, 4, 5 * R + 7
    Hq, S, scale, packed = Hkv * G, B * Hkv, 1.0 / np.sqrt(dim), (0, 2)
    pps, wide = 16, 64 + 5 * R // 8
    pages = S * 12
    i32 = lambda *s: torch.full(s, -1, dtype=torch.int32, device=DEV)  # noqa: E731
    stack, n_free = _dev(rng.permutation(pages)), _dev([pages])
    table, entries, counts = i32(S, pps), i32(S, wide, 4), torch.zeros(S, dtype=torch.int32, device=DEV)
    length, tok_off, first_pos = torch.zeros(B, dtype=torch.int32, device=DEV), i32(B + 1), i32(B)
    k_pages = torch.full((pages, R, dim), float("nan"), dtype=torch.bfloat16, device=DEV)
    v_pages = torch.full_like(k_pages, float("nan"))
    ews = torch.empty(d.dkv_page_extend_workspace_bytes(B), dtype=torch.uint8, device=DEV)
    sws = torch.empty(max(16, d.dkv_page_select_workspace_bytes(Hkv, T)), dtype=torch.uint8, device=DEV)
    rws = torch.empty(d.dkv_page_release_workspace_bytes(Hkv, pps), dtype=torch.uint8, device=DEV)
    # kept: the recent positions (the page that the next token shares among them) and an eighth of the others' runs
    keep = np.repeat(rng.uniform(size=(S, T // 8 + 1)) < 0.12, 8, axis=1)[:, :T].astype(np.uint8)
    keep[:, 2 * R:4 * R] = 0
    keep[:, T - 9:] = 1
    masks = [torch.zeros(Hkv * T + 16, dtype=torch.uint8, device=DEV)[:Hkv * T].view(Hkv, T) for _ in range(B)]
    for b in packed:
        masks[b].copy_(_dev(keep[b * Hkv:(b + 1) * Hkv], torch.uint8))
    hist = [np.zeros((2, Hkv, 0, dim)) for _ in range(B)]

    def select(b, past, used=None):
        at = slice(b * Hkv, (b + 1) * Hkv)
        d.dkv_page_select(masks[b], table[at], R, past, entries[at], counts[at], i32(Hkv), sws, page_used=used)

    def step(new, attend=True):
        tokens = sum(new)
        x = _bf16(rng, (tokens, Hq + 2 * Hkv, dim))
        xd, xn = x.to(DEV), x.double().numpy()
        slots = torch.full((tokens, Hkv), -5, dtype=torch.int64, device=DEV)
        d.dkv_page_extend(_dev(new), length, stack, n_free, table, R, Hkv, tok_off, first_pos, slots, ews, entries=entries,
                          n_entries=counts)
        at = 0
        for b, n in enumerate(new):
            add = xn[at:at + n, Hq:].reshape(n, 2, Hkv, dim).transpose(1, 2, 0, 3)
            hist[b] = np.concatenate([hist[b], add], axis=2)
            at += n
        assert length.cpu().tolist() == [h.shape[2] for h in hist] and (slots >= 0).all()
        d.dkv_paged_append(xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], slots, k_pages, v_pages)
        if not attend:
            return
        for b in packed:
            select(b, hist[b].shape[2] - T)
        assert int(counts.max()) <= wide
        ws = torch.empty(max(16, d.dkv_paged_query_workspace_bytes(B, Hq, Hkv, dim, tokens, max(new), 0)),
                         dtype=torch.uint8, device=DEV)
        out = torch.empty((tokens, Hq, dim), device=DEV)
        d.dkv_paged_query_attn(xd[:, :Hq], tok_off, first_pos, k_pages, v_pages, entries, counts, scale, out, ws, Hkv,
                               max(new))
        want, at = np.zeros((tokens, Hq, dim)), 0
        for b, n in enumerate(new):
            have = hist[b].shape[2] - n
            for t in range(n):
                for h in range(Hq):
                    see = np.ones(have + t + 1, dtype=bool)
                    if b in packed:
                        see[:T] = keep[b * Hkv + h // G] != 0
                    k, v = hist[b][:, h // G, :have + t + 1][:, see]
                    s = scale * k @ xn[at + t, h]
                    p = np.exp(s - s.max())
                    want[at + t, h] = p @ v / p.sum()
            at += n
        got = out.double().cpu().numpy().reshape(-1, dim)
        # a row's largest element errs by at most some four times the row's rms of LIMIT
        assert row_rel_err(got, want.reshape(-1, dim)) <= 16 * LIMIT

    step([T, R // 2 + 3, T], attend=False)
    for b in packed:
        used = torch.empty((Hkv, pps), dtype=torch.uint8, device=DEV)
        select(b, 0, used)
        at, before = slice(b * Hkv, (b + 1) * Hkv), int(n_free)
        d.dkv_page_release(table[at], stack, n_free, rws, keep=used)
        assert int(n_free) >= before + 2 * Hkv  # whole pages went
        gone = stack[before:int(n_free)].long()
        k_pages[gone], v_pages[gone] = float("nan"), float("nan")
    for new in ([5, 2 * R + 9, 1], [1, 1, 1], [R + 20, 3, 33], [0, 1, 7], [2, R, R]):
        step(new)
