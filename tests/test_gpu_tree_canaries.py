"""Guards around every output of the rotary, storing, tree and accepting calls:
each is carved out of a larger buffer whose 4 KiB before and after it must stay
as they were, at odd sizes, with padded rows and with slots, pages, paths and
entries outside their buffers."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"
GUARD, SENTINEL = 4096, 0xA7


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


class Room:
    """Guarded tensors: room(shape, dtype) makes one, intact() looks at them all."""

    def __init__(self):
        self.bases = []

    def __call__(self, shape, dtype, byte=0):
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        base = torch.full((2 * GUARD + n,), SENTINEL, dtype=torch.uint8, device=DEV)
        base[GUARD:GUARD + n] = byte
        self.bases.append((base, n))
        return base[GUARD:GUARD + n].view(dtype).view(shape)

    def intact(self):
        torch.cuda.synchronize()
        return all(bool((b[:GUARD] == SENTINEL).all()) and bool((b[GUARD + n:] == SENTINEL).all()) for b, n in self.bases)


def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEV, dtype=dtype)


def _rows(rng, *shape, dtype=torch.bfloat16):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(device=DEV, dtype=dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens, heads, dim, rot", [(1, 1, 8, 8), (7, 3, 80, 20), (333, 5, 64, 64), (129, 2, 256, 254)])
def test_rope(d, dtype, tokens, heads, dim, rot):
    rng, room = np.random.default_rng(tokens), Room()
    out = room((tokens, heads, dim), dtype)
    pos = _dev(rng.integers(-1, 1000, size=tokens))
    for inter in (False, True):
        d.dkv_rope(_rows(rng, tokens, heads, dim, dtype=dtype), pos, torch.ones(rot // 2, device=DEV), rot, out, interleaved=inter)
        assert room.intact()


def _cache(room, fmt, pages, R, dim):
    kind = torch.float8_e4m3fn if fmt == "f8" else torch.bfloat16
    k, v = room((pages, R, dim), kind), room((pages, R, dim), kind)
    return k, v, room((pages, R, 2), torch.uint8) if fmt == "f8" else None


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_store_and_load(d, fmt, dim):
    """Slots of the pool's first and last rows, and a step outside on either side."""
    for tokens, Hq, Hkv in ((1, 1, 1), (61, 6, 3), (500, 8, 2)):
        rng, room = np.random.default_rng(tokens), Room()
        pages, R = 9, 64
        k, v, ex = _cache(room, fmt, pages, R, dim)
        slots = rng.choice(pages * R, size=(tokens, Hkv), replace=tokens * Hkv > pages * R)
        slots.reshape(-1)[::7] = rng.choice([0, pages * R - 1, -1, pages * R, 1 << 40, -(1 << 40)], size=len(slots.reshape(-1)[::7]))
        q_out = room((tokens, Hq, dim), torch.bfloat16)
        x = _rows(rng, tokens, Hq + 2 * Hkv, dim)
        pos = _dev(rng.integers(-1, 10000, size=tokens))
        d.dkv_paged_store(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], _dev(slots, torch.int64), k, v, scales=ex, q=x[:, :Hq], q_out=q_out,
                          pos=pos, inv_freq=torch.ones(dim // 2, device=DEV), rot_dim=dim)
        assert room.intact(), "dkv_paged_store wrote outside"
        ko, vo = (room((tokens, Hkv, dim), torch.bfloat16) for _ in range(2))
        d.dkv_paged_load(_dev(slots, torch.int64), k, v, ko, vo, scales=ex)
        assert room.intact(), "dkv_paged_load wrote outside"


@pytest.mark.parametrize("sizes, pad, words", [([1], 0, 1), ([70, 0, 5], 3, 2), ([1000, 24], 1, 17)])
def test_tree_plan(d, sizes, pad, words):
    rng, room = np.random.default_rng(words), Room()
    tokens = sum(sizes) + pad
    pos, mask = room((tokens,), torch.int32), room((tokens, words), torch.int64)
    off, first = _dev(np.concatenate([[0], np.cumsum(sizes)])), _dev(rng.integers(0, 2 ** 31 - 1, size=len(sizes)))
    for parent in (None, _dev(rng.integers(-2 ** 31, 2 ** 31 - 1, size=tokens)), _dev(np.arange(tokens) // 2 - 1)):
        d.dkv_tree_plan(off, first, max(sizes), pos, parent=parent, mask=mask)
        assert room.intact()


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("G", [1, 7, 16])
def test_tree_attention(d, fmt, dim, G):
    """Every kernel's shape: few and many query rows, short and long lists, split over workgroups or not."""
    Hkv, R, pages, B = 2, 32, 40, 3
    for new, hint in (([1, 1, 1], 0), ([3, 0, 5], 1000), ([9, 17, 2], 1 << 20), ([40, 3, 64], 0), ([90, 1, 60], 1 << 22)):
        rng, room = np.random.default_rng(sum(new)), Room()
        k, v, ex = _cache(room, fmt, pages, R, dim)
        tokens, most = sum(new) + 2, max(new)
        out = room((tokens, Hkv * G, dim), torch.float32)
        fmt_code = d.DKV_CACHE_F8 if fmt == "f8" else d.DKV_CACHE_BF16
        ws = room((max(16, d.dkv_paged_tree_workspace_bytes(fmt_code, B, Hkv * G, Hkv, dim, tokens, most, hint)),), torch.uint8, 0xFF)
        entries = np.full((B * Hkv, 12, 4), -1)
        for s in range(B * Hkv):
            entries[s, :, 0] = rng.integers(-1, pages + 1, size=12)   # a page outside is no entry
            entries[s, :, 1] = np.arange(12)
            entries[s, :, 2] = rng.integers(0, 5, size=12)
            entries[s, :, 3] = rng.integers(20, R + 1, size=12)
        mask = _dev(rng.integers(-2 ** 63, 2 ** 63 - 1, size=(tokens, -(-most // 64))), torch.int64)
        for m in (mask, None):
            d.dkv_paged_tree_attn(_rows(rng, tokens, Hkv * G, dim), _dev(np.concatenate([[0], np.cumsum(new)])), _dev([300, -1, 7]),
                                  k, v, _dev(entries), _dev([12, 12, 0, 5, 30, -3]), 0.1, out, ws, Hkv, most, mask=m, scales=ex,
                                  rows_hint=hint)
            assert room.intact(), (new, hint)
            assert (out[-2:] == 0).all()  # nobody's rows, as they were


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
def test_accept(d, fmt):
    rng, room = np.random.default_rng(4), Room()
    N, B, Hkv, R, dim, pps, pages, most = 6, 3, 2, 32, 64, 5, 20, 64
    k, v, ex = _cache(room, fmt, pages, R, dim)
    new_len, keep = room((N,), torch.int32), room((N * Hkv, pps), torch.uint8)
    for _ in range(4):
        first = rng.choice([0, 31, 32, 100, pps * R - 1, pps * R, 2 ** 31 - 1, -1], size=N)
        path = np.sort(rng.integers(-1, 200, size=(B, most)), axis=1)
        path[0] = np.arange(most) + 2
        d.dkv_paged_accept(_dev(first), _dev(path), _dev(rng.integers(-1, most + 2, size=B)),
                           _dev(rng.integers(-1, pages + 1, size=(N * Hkv, pps))), Hkv, k, v, new_len, scales=ex, keep=keep)
        assert room.intact()
