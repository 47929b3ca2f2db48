"""What the binding makes of the arguments of the calls that fill a paged cache and attend chunks over it."""

import numpy as np
import pytest
import torch

from test_gpu_paged_query import DEV, Batch, _dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


def _calls(d):
    """Each of the calls on small tensors, as a function of its stream."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    ws, slots = torch.empty(4096, dtype=torch.uint8, device=DEV), torch.zeros((4, 2), dtype=torch.int64, device=DEV)
    pool, x = torch.zeros((3, 32, 64), dtype=torch.bfloat16, device=DEV), torch.zeros(
        (4, 2, 64), dtype=torch.bfloat16, device=DEV)
    b = Batch(np.random.default_rng(1), [40], [3], 2, 4, 64, 32)
    return [lambda s: d.dkv_page_extend(i32(2), i32(2), i32(9), i32(1), i32(4, 3), 32, 2, i32(3), i32(2), slots, ws, stream=s),
            lambda s: d.dkv_page_release(i32(4, 3), i32(9), i32(1), ws, stream=s),
            lambda s: d.dkv_paged_append(x, x, slots, pool, pool, stream=s),
            lambda s: b.run(d, stream=s)]


class _StreamOf:
    def __init__(self, device_index):
        self.device_index, self.cuda_stream = device_index, 0


@pytest.mark.parametrize("call", range(4))
def test_another_device_is_refused(d, call, monkeypatch):
    """Tensors that are not on the current device, or a stream that is not: a launch would go to the wrong one."""
    f = _calls(d)[call]
    f(None)
    f(torch.cuda.current_stream())
    with pytest.raises(ValueError, match="current device"):
        f(_StreamOf(torch.cuda.current_device() + 1))
    monkeypatch.setattr(d.binding, "_current_device", lambda: torch.cuda.current_device() + 1)
    with pytest.raises(ValueError, match="current device"):
        f(None)
    torch.cuda.synchronize()


def test_a_longest_chunk_beyond_int32_is_all_tokens(d):
    x = Batch(np.random.default_rng(2), [300, 90], [80, 3], 2, 4, 64, 32)
    want = x.run(d)
    x.max_q = 1 << 32
    assert torch.equal(x.run(d), want)
