"""Quantised rows of V whose exponent byte is below 67, the least that
dkv_paged_store writes: a row of zeros is the same row with any byte, and the
share of its key in the softmax's sum must not depend on it.  Other writers of
the format take the smallest exponent that holds a row, down to byte 10.
Tolerance: test_gpu_tree_attn.py's."""

import numpy as np
import pytest
import torch

from test_gpu_tree_attn import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


# query rows (4 a token), and hints that choose the kernel: the short ones' forms, query tiles with
# two key halves (up to 128 rows) and without
FORMS = [(1, 100), (5, 100), (12, 100), (30, 1000), (30, 1 << 20), (50, 20000), (50, 1 << 20), (100, 1 << 20)]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n, hint", FORMS)
@pytest.mark.parametrize("low", [0, 10, 66])
def test_rows_of_zeros_with_any_exponent(d, dim, n, hint, low):
    rng = np.random.default_rng([dim, n, low])
    b = Batch(rng, "f8", [900, 3], [n, 1], 2, 4, dim, 64, kscale=1.5, vsizes=(0.0, 0.0, 0.0, 100.0))
    zeros = torch.from_numpy((b.v == 0).all(axis=2)).to(b.scales.device)
    assert zeros.float().mean() > 0.1
    exps = b.scales[..., 1]
    exps[zeros] = low if low else torch.randint(0, 67, exps[zeros].shape, dtype=torch.uint8, device=exps.device)
    b.check(d, scale=0.5, hint=hint)


@pytest.mark.parametrize("n, hint", FORMS)
def test_tiny_rows(d, n, hint):
    """Rows below 448 * 2^-60 count as codes times 2^-60: within 2^-51 of what they are, far below the others' rounding."""
    rng = np.random.default_rng(n)
    b = Batch(rng, "f8", [900, 3], [n, 1], 2, 4, 128, 64, kscale=1.5, vsizes=(1.0, 2.0 ** -70, 30.0))
    small = torch.from_numpy(np.nan_to_num(np.abs(b.v)).max(axis=2) < 2.0 ** -51).to(b.scales.device)
    written = torch.from_numpy(np.isfinite(b.v).all(axis=2)).to(b.scales.device)
    b.scales[..., 1][small & written] = 40
    b.check(d, scale=0.5, hint=hint)


@pytest.mark.parametrize("n, hint", FORMS)
def test_nothing_but_zeros_with_the_least_byte(d, n, hint):
    rng = np.random.default_rng(n)
    b = Batch(rng, "f8", [300], [n], 2, 4, 64, 32, vsizes=(0.0,))
    b.scales[..., 1] = torch.where(torch.from_numpy(np.isfinite(b.v).all(axis=2)).cuda(), 0, 255).to(torch.uint8)
    assert (b.check(d, hint=hint) == 0).all()
