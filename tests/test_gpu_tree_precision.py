"""dkv_paged_tree_attn against float64 in the outputs' own norms, in every form
that its kernels have: both formats and head sizes, with and without a mask,
blocks of few and many rows in the short kernels and in query tiles (with two key
halves and without), unsplit and split over long segments.  The bound tells
the parts that a weight enters its product in: a quantised cache has two of fp16
(one would err by more than a hundred times the limit), bf16 pools have three
(two would err by twice the limit).  The limit is derived in
test_paged_precision_cpu.py, for values of equal spread, as here; sequences are
checked one by one, by the mean square of their rows' errors."""

import numpy as np
import pytest
import torch

from test_gpu_tree_attn import KEEP, Batch
from test_paged_precision_cpu import LIMIT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


def _check(d, x, **kw):
    got, (want, _, _) = x.run(d, **kw).double().cpu().numpy(), x.want()
    assert (got[want == KEEP] == KEEP).all() and np.isfinite(got).all()
    for b, (lo, hi) in enumerate(zip(x.tok_off[:-1], x.tok_off[1:])):
        rows = [y[lo:hi].reshape(-1, x.dim) for y in (got, want)]
        err = np.linalg.norm(rows[0] - rows[1], axis=1) / np.linalg.norm(rows[1], axis=1)
        assert np.sqrt((err ** 2).mean()) <= LIMIT, (b, x.new[b], np.sqrt((err ** 2).mean()))


FMTS = ["f8", "bf16"]
# tokens of four rows each, and hints of the rows that all segments hold: few, as many as there are, and many
# (which send blocks of 33 to 256 rows to the query tiles)
BLOCKS = [(1, None), (4, None), (5, None), (8, None), (9, None), (15, None), (15, 1 << 20), (25, None), (25, 1 << 20),
          (32, 1 << 20), (33, None), (50, None), (50, 1 << 20), (64, 1 << 20), (75, None), (100, None)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("mask", [None, "tree"])
@pytest.mark.parametrize("new, hint", BLOCKS)
def test_blocks(d, fmt, dim, mask, new, hint):
    rng = np.random.default_rng([dim, new])
    _check(d, Batch(rng, fmt, [3000, 700], [new, max(1, new // 2)], 2, 4, dim, 64, mask=mask, vsizes=(1.0,)), hint=hint)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 6, 16, 30, 64, 150])
def test_long_segments(d, fmt, dim, new):
    """20,000 keys cut into ranges over the whole card and joined; a hint that is far too small, so that few workgroups
    or one take them."""
    rng = np.random.default_rng([dim, new])
    x = Batch(rng, fmt, [20000, 3000], [new, max(1, new // 2)], 1, 4, dim, 128, mask="tree", vsizes=(1.0,))
    for hint in (None, 3000):
        _check(d, x, hint=hint)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new, hint", [(15, 1 << 17), (15, 1), (30, 1), (30, 1 << 19), (60, 1 << 20), (70, 1 << 20)])
def test_many_segments(d, fmt, dim, new, hint):
    """72 segments: the quantised tiles from 33 rows on; whole units without a split."""
    rng = np.random.default_rng([dim, new])
    held = rng.integers(40, 300, size=9)
    _check(d, Batch(rng, fmt, held, rng.integers(1, new + 1, size=9), 8, 4, dim, 32, mask="tree", vsizes=(1.0,)), hint=hint)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [2, 20, 60, 90])
def test_selected_runs(d, fmt, dim, new):
    rng = np.random.default_rng([dim, new])
    _check(d, Batch(rng, fmt, [4000, 2500], [new, 3], 2, 4, dim, 128, keep=0.4, mask="tree", vsizes=(1.0,)))
