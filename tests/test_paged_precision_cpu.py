"""How far attention is off when a probability enters its product with V as one,
two or three bf16 parts, in float64 on the host, and the limit that
tests/test_gpu_paged_precision.py holds the kernels to.

A part is the bf16 rounding of what the parts before it left out, so one part
misses p by up to 2^-8 p, two by up to 2^-17 p and three by up to 2^-26 p, less
than fp32's own 2^-24.  An output row sum_i p_i v_i / sum_i p_i of values of
equal spread errs by sqrt(sum (d_i p_i)^2 / sum p_i^2) of its norm, d_i the
relative miss of p_i: a mean of the misses, at any number of keys."""

import numpy as np
import pytest
import torch

# of the outputs' norm.  Half of what two parts err by and above the fp32
# operations' errors, in quadrature: the exponent's argument, below 16, off by up
# to 2^-21 (1.9e-7 of a probability, rms); scores of some 128 products 1e-7 to 3e-7;
# the exponential 5e-8; output sums of up to 400 additions, each off by 2.4e-8 of
# the sum so far, 3.3e-7: 5e-7.
LIMIT = 1e-6


def parts_of(p, n):
    """Sum of the first n bf16 parts of float32 values, as float64."""
    left, total = p.clone(), torch.zeros_like(p, dtype=torch.float64)
    for _ in range(n):
        part = left.to(torch.bfloat16).to(torch.float32)
        total += part.double()
        left = left - part  # exact: the remainder of a rounding fits
    return total


@pytest.mark.parametrize("keys", [100, 1000, 40000])
@pytest.mark.parametrize("dim", [64, 128])
def test_the_limit_tells_the_parts_apart(keys, dim):
    gen = torch.Generator().manual_seed(keys + dim)
    f = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64).bfloat16().double()  # noqa: E731
    q, k, v = f(16, dim), f(keys, dim), f(keys, dim)
    s = q @ k.T / np.sqrt(dim)
    p = torch.exp(s - s.amax(dim=1, keepdim=True)).float()
    want = p.double() @ v
    err = [float((parts_of(p, n) @ v - want).norm() / want.norm()) for n in (1, 2, 3)]
    assert err[0] > 500 * LIMIT and err[1] > 1.8 * LIMIT and err[2] < LIMIT / 20, err
