"""A rotated bf16 value is rounded once from 64 bits to fp32 and from there to
bf16: bit for bit the oracle's, but where the two sides' own errors in 64 bits,
below 2^-47 (|a| + |b|) mscale together, leave open on which side of a border a
value lies.  (Products in fp32 put some 5 of 192,000 values on the other side,
bf16 cut instead of rounded every second one.)"""

import numpy as np
import pytest
import torch

from oracle import tree_cache as tc

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEV, dtype=dtype)


def _bf16(x):
    return torch.from_numpy(x.astype(np.float32)).bfloat16().double().numpy()


def _both(x, rot, inter):
    """|a| + |b| of the pair that an element belongs to, zero for those that stay."""
    y, n, out = np.abs(x), rot // 2, np.zeros_like(x)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if inter else (slice(0, n), slice(n, 2 * n))
    out[..., a] = out[..., b] = y[..., a] + y[..., b]
    return out


def _check(got, x, pos, f, rot, inter, ms):
    want = tc.rope(x, pos, f, rot, inter, ms)
    open_ = 2.0 ** -47 * ms * _both(x, rot, inter)
    low, high = _bf16(want - open_), _bf16(want + open_)
    np.testing.assert_array_equal(np.where(got == high, high, low), got)
    assert (low != high).mean() < 1e-4  # hardly any is left open


def _inputs(rng, tokens, heads, dim, rot):
    x = torch.from_numpy(rng.standard_normal((tokens, heads, dim)).astype(np.float32)).bfloat16()
    pos = rng.integers(0, 131072, size=tokens)
    pos[0] = 0
    f = (10000.0 ** (-np.arange(rot // 2) / (rot // 2)) * rng.uniform(0.9, 1.1, rot // 2)).astype(np.float32)
    return x, pos, f


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dim, rot", [(128, 128), (128, 96), (128, 22), (64, 64), (80, 80), (256, 200)])
@pytest.mark.parametrize("ms", [1.0, 1.2079441])
def test_rope(d, dim, rot, inter, ms):
    rng = np.random.default_rng([dim, rot, inter])
    x, pos, f = _inputs(rng, 120, 20, dim, rot)
    out = torch.zeros_like(x, device=DEV)
    d.dkv_rope(x.to(DEV), _dev(pos), _dev(f, torch.float32), rot, out, interleaved=inter, mscale=ms)
    _check(out.double().cpu().numpy(), x.double().numpy(), pos, f, rot, inter, float(np.float32(ms)))


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dim, rot", [(128, 128), (128, 64), (64, 64), (64, 18)])
@pytest.mark.parametrize("tokens, Hq, Hkv", [(3, 4, 2), (100, 12, 8), (2100, 2, 1)])
def test_store(d, dim, rot, inter, tokens, Hq, Hkv):
    """Queries, and keys in the pool, of one launch; V's rows are copied."""
    rng = np.random.default_rng([dim, rot, inter, tokens])
    x, pos, f = _inputs(rng, tokens, Hq + 2 * Hkv, dim, rot)
    R = 64
    pages = tokens * Hkv // R + 2
    slots = rng.permutation(pages * R)[:tokens * Hkv].reshape(tokens, Hkv)
    k, v = (torch.zeros((pages, R, dim), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q_out = torch.zeros((tokens, Hq, dim), dtype=torch.bfloat16, device=DEV)
    y = x.to(DEV)
    d.dkv_paged_store(y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:], _dev(slots, torch.int64), k, v, q=y[:, :Hq], q_out=q_out, pos=_dev(pos),
                      inv_freq=_dev(f, torch.float32), rot_dim=rot, interleaved=inter, mscale=1.1)
    ms, x64 = float(np.float32(1.1)), x.double().numpy()
    _check(q_out.double().cpu().numpy(), x64[:, :Hq], pos, f, rot, inter, ms)
    _check(k.view(-1, dim)[torch.from_numpy(slots).to(DEV)].double().cpu().numpy(), x64[:, Hq:Hq + Hkv], pos, f, rot, inter, ms)
    assert torch.equal(v.view(-1, dim)[torch.from_numpy(slots).to(DEV)], y[:, Hq + Hkv:])
