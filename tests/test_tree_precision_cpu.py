"""How far attention over quantised rows is off when a weight enters its product
with V's codes as one or two fp16 parts, in float64 on the host, with the limit
of test_paged_precision_cpu.py: the same fp32 operations stand behind it, and
what two parts leave out is below them.

A part is cut (not rounded) to 11 bits: one misses a weight by up to 2^-10 of
itself, two by up to 2^-21."""

import numpy as np
import pytest
import torch

from oracle import tree_cache as tc
from test_paged_precision_cpu import LIMIT


def cut(x):
    """float32 values towards zero to fp16, as float64 (values within fp16's normal range)."""
    return (x.view(torch.int32) & ~0x1FFF).view(torch.float32).double()


def parts_of(w, n):
    total, left = torch.zeros_like(w, dtype=torch.float64), w.clone()
    for _ in range(n):
        total += cut(left)
        left = (w.double() - total).float()  # exact: what a cut leaves out fits
    return total


@pytest.mark.parametrize("keys", [100, 1000, 40000])
@pytest.mark.parametrize("dim", [64, 128])
def test_the_limit_tells_the_parts_apart(keys, dim):
    rng = np.random.default_rng(keys + dim)
    q = torch.from_numpy(rng.standard_normal((16, dim)))
    k, v = (torch.from_numpy(tc.row_values(*tc.quantise(rng.standard_normal((keys, dim))))) for _ in range(2))
    s = q @ k.T / np.sqrt(dim)
    p = torch.exp(s - s.amax(dim=1, keepdim=True)).float() * 2.0 ** 7  # raised clear of fp16's subnormals, as the kernels do
    want = p.double() @ v
    err = [float((parts_of(p, n) @ v - want).norm() / want.norm()) for n in (1, 2)]
    assert err[0] > 100 * LIMIT and err[1] < LIMIT / 3, err
