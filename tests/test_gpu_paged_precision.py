"""A probability enters its product with V as three bf16 parts, 24 bits, at every
length and in every form of dkv_paged_query_attn: every sequence's outputs
against float64, row by row in the rows' own norms, below what two parts would
give."""

import numpy as np
import pytest
import torch

from test_gpu_paged_query import KEEP, Batch
from test_paged_precision_cpu import LIMIT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


def _check(d, x, **kw):
    got, want = x.run(d, **kw).double().cpu().numpy(), x.want()
    assert (got[want == KEEP] == KEEP).all() and np.isfinite(got).all()
    for b, (lo, hi) in enumerate(zip(x.tok_off[:-1], x.tok_off[1:])):
        rows = [y[lo:hi].reshape(-1, x.dim) for y in (got, want)]
        err = np.linalg.norm(rows[0] - rows[1], axis=1) / np.linalg.norm(rows[1], axis=1)
        assert np.sqrt((err ** 2).mean()) <= LIMIT, (b, x.new[b], np.sqrt((err ** 2).mean()))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("G,new", [(4, 1), (4, 8), (4, 15), (4, 30), (8, 30)])
@pytest.mark.parametrize("held", [90, 1000, 20000])
def test_short_blocks(d, dim, G, new, held):
    """8 to 240 query rows per segment: the kernels for short blocks, unsplit and split."""
    rng = np.random.default_rng([dim, G, new, held])
    _check(d, Batch(rng, [held, held // 2], [new, new], 1, G, dim, 64))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("held,hint", [(20, None), (1000, 1), (4000, None), (32768 - 70, None), (33000, None), (60000, None)])
def test_query_tiles(d, dim, held, hint):
    """More rows than short blocks have: one workgroup per tile, and slices, around 32,768 rows and beyond."""
    rng = np.random.default_rng([dim, held])
    _check(d, Batch(rng, [held, 40], [20, 17], 1, 16, dim, 256), hint=hint)


@pytest.mark.parametrize("dim,G,B,new,held", [(64, 16, 40, 320, 700), (128, 7, 64, 290, 500)])
def test_whole_tiles(d, dim, G, B, new, held):
    rng = np.random.default_rng([dim, B, held])
    new = rng.integers(new - 60, new + 1, size=B)
    _check(d, Batch(rng, rng.integers(held - 100, held + 1, size=B), new, 1, G, dim, 128))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [3, 20])
def test_few_keys_in_many_large_pages(d, dim, new):
    """A selection's short runs, one in each of 40 pages of 1,024 rows: some 1,200 keys among 40,960 rows."""
    rng = np.random.default_rng([dim, new])
    x = Batch(rng, [40 * 1024, 30 * 1024], [new, 3], 1, 16, dim, 1024)
    lo = rng.integers(0, 1024 - 30, size=(2, 40))
    for s, n in enumerate((40, 30)):
        x.entries[s, :n, 2], x.entries[s, :n, 3] = lo[s, :n], lo[s, :n] + 30
    _check(d, x)
