"""Tree calls whose inputs and outputs are neighbouring parts of one buffer: what
the refusal of shared bytes must leave alone."""

import numpy as np
import pytest
import torch

from oracle import tree_cache as tc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


def _parts(*arrays):
    """int32 arrays side by side in one device buffer, as views of it."""
    whole = torch.from_numpy(np.concatenate([a.reshape(-1) for a in arrays]).astype(np.int32)).cuda()
    out, at = [], 0
    for a in arrays:
        out.append(whole[at:at + a.size].view(a.shape))
        at += a.size
    return out


def test_accept_takes_neighbouring_parts(d):
    rng = np.random.default_rng(3)
    B, layers, Hkv, R, dim, pps = 3, 2, 2, 32, 64, 3
    N, pages = B * layers, B * layers * Hkv * pps
    table = rng.permutation(pages).reshape(N * Hkv, pps)
    first = np.tile(rng.integers(0, 40, size=B), layers)
    path = np.sort(np.stack([rng.permutation(20)[:6] for _ in range(B)]), axis=1)
    n_path = np.array([6, 0, 3])
    k, v = (torch.from_numpy(rng.standard_normal((pages, R, dim)).astype(np.float32)).bfloat16().cuda() for _ in range(2))
    before = [x.float().cpu().numpy() for x in (k, v)]
    f, new_len, p, n, t = _parts(first, np.zeros(N), path, n_path, table)
    keep = torch.ones((N * Hkv, pps), dtype=torch.uint8, device="cuda")
    d.dkv_paged_accept(f, p, n, t, Hkv, k, v, new_len, keep=keep)
    pools, want, wk = tc.accept(first, path, n_path, table, R, Hkv, before)
    assert new_len.tolist() == want and keep.tolist() == wk.tolist()
    for got, x in zip((k, v), pools):
        assert np.array_equal(got.float().cpu().numpy(), x)
    assert f.tolist() == first.tolist() and p.tolist() == path.tolist() and t.tolist() == table.tolist()
    with pytest.raises(d.DkvError):
        d.dkv_paged_accept(f, p, n, t, Hkv, k, v, f, keep=keep)


def test_plan_takes_the_parents_place_and_neighbouring_parts(d):
    rng = np.random.default_rng(4)
    new = np.array([5, 0, 70, 1, 33])
    tokens, words = int(new.sum()) + 3, 2
    off = np.concatenate([[0], np.cumsum(new)])
    first = np.array([7, 3, 0, 500, -1])
    parent = rng.integers(-2, 40, size=tokens)
    want, bits = tc.tree_plan(off, first, 70, tokens, parent, words)
    o, f, p, pos = _parts(off, first, parent, np.zeros(tokens))
    for at in (pos, p):
        mask = torch.zeros((tokens, words), dtype=torch.int64, device="cuda")
        d.dkv_tree_plan(o, f, 70, at, parent=p, mask=mask)
        assert at.tolist() == want.tolist() and np.array_equal(mask.cpu().numpy(), bits.view(np.int64))
        assert o.tolist() == off.tolist() and f.tolist() == first.tolist()
