"""Quantised attention: how small a share of the softmax's sum still counts when
rows of V lie as far apart as the format's range for it allows (2^-60 and 2^17 a
code).  A weight's reference carries V's exponent, so a key of zeros in V is
2^77 further down than its probability says.

The call is one workgroup's: 2^24 keys of probability 2^-41 of the largest, all of
zeros in V, behind some of 2^-49 that set the running maximum (which moves only
when passed by more than 2^8), and the largest, of 2^24.9 in V, at the very end.
Then the reference moves by 126, the most that fp32's exponential has.  The
2^24 keys together are 2^-17 of the sum.

Tolerance, of the output: a lane's keys add up exactly (equal powers of two); the
lanes, waves and key halves, at most 32 of a row, are joined by as many
additions next to one, each off by 2^-25 at most; the division, the weight's parts and
the product's rounding together 2^-22: 2^-19.7, so 2^-19, a quarter of what would be lost."""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"
R, FULL = 1024, 1 << 14  # rows of a page, pages of the request


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 5, 15, 25, 50, 75])  # four rows each: every form that takes a call whole
def test_shares_down_to_2_41(d, dim, n):
    f8 = torch.float8_e4m3fn
    k, v = (torch.zeros((4, R, dim), device=DEV) for _ in range(2))
    ex = torch.full((4, R, 2), 127, dtype=torch.uint8, device=DEV)
    ex[..., 1] = 67
    k[0, :, 0] = -8.0                      # the first keys, 2^-49
    k[2, R - 1, 0], k[2, R - 1, 1] = 40.0, 1.0  # the last, 2^41 times the others'
    v[2, R - 1], ex[2, R - 1, 1] = 240.0, 127 + 17
    entries = torch.zeros((1, FULL + 1, 4), dtype=torch.int32, device=DEV)
    entries[0, :, 0] = 1
    entries[0, 0, 0], entries[0, FULL - 1, 0], entries[0, FULL, 0] = 0, 2, 3
    entries[0, :, 1] = torch.arange(FULL + 1)
    entries[0, :, 3] = R
    entries[0, FULL, 3] = n
    q = torch.zeros((n, 4, dim), dtype=torch.bfloat16, device=DEV)
    q[..., :2] = 1.0
    out = torch.zeros((n, 4, dim), device=DEV)
    off, first = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, n], [FULL * R]))
    count = torch.full((1,), FULL + 1, dtype=torch.int32, device=DEV)
    assert d.dkv_paged_tree_workspace_bytes(d.DKV_CACHE_F8, 1, 4, 1, dim, n, n, 1) == 0  # one workgroup's
    d.dkv_paged_tree_attn(q, off, first, k.to(f8), v.to(f8), entries, count, math.log(2.0), out, None, 1, n, scales=ex,
                          rows_hint=1)
    scale = float(np.float32(math.log(2.0))) / math.log(2.0)
    seen = np.arange(1, n + 1)[:, None, None]  # of the new tokens, of the middle ones' probability
    middle, low = 2.0 ** (-41 * scale), 2.0 ** (-49 * scale)
    want = 240.0 * 2.0 ** 17 / (1.0 + ((FULL - 1) * R - 1 + seen) * middle + R * low)
    err = np.abs(out.double().cpu().numpy() / want - 1).max()
    assert err <= 2.0 ** -19, err * 2.0 ** 19
