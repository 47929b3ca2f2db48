"""Filling a paged cache, on the host: the oracle's results worked out by hand
for small cases, and the entry points' refusals (no call passes validation, so
nothing reaches a GPU)."""

import ctypes

import numpy as np
import pytest

import oracle as o
import paper_2609_32663_amd as d
from oracle import page_fill as pf

A = ctypes.c_void_p(0x10000)    # fake 16-byte-aligned device address
MIS = ctypes.c_void_p(0x10008)  # 8-byte-aligned only
ODD = ctypes.c_void_p(0x10002)
NUL = None


# ---------------------------------------------------------------------------
# the oracle
# ---------------------------------------------------------------------------

def test_extend_by_hand():
    """Two KV heads, pages of 32: a request that fills its page and starts another, one that starts from nothing, one
    that needs no page and one for which the stack is too low."""
    table = np.full((8, 3), -1, dtype=np.int32)
    table[0, 0], table[1, 0] = 50, 51
    table[4, 0], table[5, 0] = 60, 61
    got = pf.page_extend([3, 40, 1, 33], [31, 0, 5, 0], [7, 6, 5, 4, 3, 2, 1], table, 32, 2, 80)
    assert got["needed"] == 2 + 4 + 0 + 4 and got["stack"] == [7]
    np.testing.assert_array_equal(got["tok_off"], [0, 3, 43, 44, 77])
    np.testing.assert_array_equal(got["first_pos"], [31, 0, 5, -1])
    np.testing.assert_array_equal(got["new_len"], [34, 40, 6, 0])
    np.testing.assert_array_equal(got["table"], [[50, 1, -1], [51, 2, -1], [3, 4, -1], [5, 6, -1], [60, -1, -1],
                                                 [61, -1, -1], [-1, -1, -1], [-1, -1, -1]])
    np.testing.assert_array_equal(got["slots"][:3], [[50 * 32 + 31, 51 * 32 + 31], [32, 64], [33, 65]])
    np.testing.assert_array_equal(got["slots"][[3, 34, 35, 42]], [[96, 160], [127, 191], [128, 192], [135, 199]])
    np.testing.assert_array_equal(got["slots"][43], [60 * 32 + 5, 61 * 32 + 5])
    assert (got["slots"][44:] == -1).all()


def test_release_by_hand():
    table, stack = pf.page_release(np.array([[4, -1, 9], [2, 3, -1]]), np.array([[1, 0, 0], [0, 0, 0]]), [8], 3)
    np.testing.assert_array_equal(table, [[4, -1, -1], [-1, 3, -1]])  # no room for page 3
    assert stack == [8, 9, 2]


def test_chunk_attention_is_the_packed_query_block():
    """A chunk over the entries of a selection equals the oracle's query block over the packed cache."""
    rng = np.random.default_rng(3)
    T, R, n_q, Hkv, G, dim = 150, 32, 9, 2, 3, 64
    f = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    k, v, kn, vn, q = f(1, Hkv, T, dim), f(1, Hkv, T, dim), f(Hkv, n_q, dim), f(Hkv, n_q, dim), f(1, n_q, Hkv * G, dim)
    mask = (rng.uniform(size=(1, Hkv, T)) < 0.4).astype(np.uint8)
    ref = o.compact(k, v, mask, n_q)
    kc, vc = o.append(ref["k_c"], ref["v_c"], ref["seg_off"], ref["seg_len"], kn.reshape(1, Hkv, n_q, dim),
                      vn.reshape(1, Hkv, n_q, dim), 0)
    want = o.query_attn(q, kc, vc, ref["seg_off"], ref["seg_len"], 0, 0.1, Hkv, o.F32)
    pps = -(-(T + n_q) // R)
    table = rng.permutation(Hkv * pps).reshape(Hkv, pps)
    pools = []
    for x, new in ((k, kn), (v, vn)):
        whole = np.zeros((Hkv, pps * R, dim), dtype=np.float32)
        whole[:, :T + n_q] = np.concatenate([x[0], new], axis=1)
        pool = np.zeros((Hkv * pps, R, dim), dtype=np.float32)
        pool[table] = whole.reshape(Hkv, pps, R, dim)
        pools.append(pool)
    sel = o.page_select(mask[0], table, R, n_q)
    got = pf.chunk_attn(q[0], [0, n_q], [T], pools[0], pools[1], sel["entries"], sel["n_entries"], 0.1, Hkv, o.F32, n_q)
    np.testing.assert_allclose(got, want[0], rtol=1e-12, atol=1e-13)


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------

def test_extend_validation():
    lib, ws = d.library(), d.dkv_page_extend_workspace_bytes(4)
    assert ws > 0 and d.dkv_page_extend_workspace_bytes(-1) == 0

    def call(N=4, Hkv=2, R=128, new=A, length=A, new_len=A, free=A, cap=10, nf=A, nfo=A, table=A, pps=3, off=A, pos=A,
             slots=A, most=100, ent=NUL, ne=NUL, max_e=0, needed=NUL, w=A, w_bytes=ws):
        return lib.dkv_page_extend(N, Hkv, R, new, length, new_len, free, cap, nf, nfo, table, pps, off, pos, slots, most,
                                   ent, ne, max_e, needed, w, w_bytes, NUL)

    for bad in (dict(N=-1), dict(Hkv=0), dict(pps=-1), dict(most=-1), dict(cap=-1), dict(max_e=-1), dict(new=NUL),
                dict(length=NUL), dict(new_len=NUL), dict(free=NUL), dict(nf=NUL), dict(nfo=NUL), dict(table=NUL),
                dict(off=NUL), dict(pos=NUL), dict(slots=NUL), dict(max_e=3)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    for bad in (dict(R=100), dict(R=16), dict(R=2048), dict(N=8192, Hkv=8, w_bytes=1 << 20), dict(Hkv=4, most=1 << 30),
                dict(Hkv=1, most=(1 << 31) - 127)):
        assert call(**bad) == d.DKV_ERR_UNSUPPORTED, bad
    assert call(ent=MIS, max_e=3) == d.DKV_ERR_MISALIGNED
    assert call(slots=ODD) == d.DKV_ERR_MISALIGNED
    for bad in (dict(w=NUL), dict(w=ODD), dict(w_bytes=ws - 1)):
        assert call(**bad) == d.DKV_ERR_WORKSPACE, bad


def test_release_validation():
    lib, ws = d.library(), d.dkv_page_release_workspace_bytes(4, 100)
    assert ws > 0 and d.dkv_page_release_workspace_bytes(-1, 3) == 0

    def call(nseg=4, pps=100, table=A, keep=NUL, out=A, free=A, cap=10, nf=A, nfo=A, w=A, w_bytes=ws):
        return lib.dkv_page_release(nseg, pps, table, keep, out, free, cap, nf, nfo, w, w_bytes, NUL)

    for bad in (dict(nseg=-1), dict(pps=-1), dict(cap=-1), dict(table=NUL), dict(out=NUL), dict(free=NUL), dict(nf=NUL),
                dict(nfo=NUL)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    assert call(nseg=65536, pps=32768) == d.DKV_ERR_UNSUPPORTED
    for bad in (dict(w=NUL), dict(w=ODD), dict(w_bytes=ws - 1)):
        assert call(**bad) == d.DKV_ERR_WORKSPACE, bad


def test_paged_append_validation():
    lib = d.library()

    def call(dtype=d.DKV_BF16, n=4, Hkv=2, dim=128, kn=A, vn=A, stride=256, slots=A, k=A, v=A, pages=10, R=128):
        return lib.dkv_paged_append(dtype, n, Hkv, dim, kn, vn, stride, slots, k, v, pages, R, NUL)

    for bad in (dict(dtype=2), dict(n=-1), dict(Hkv=0), dict(pages=-1), dict(stride=255), dict(stride=1 << 31), dict(kn=NUL),
                dict(vn=NUL), dict(slots=NUL), dict(k=NUL), dict(v=NUL)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    for bad in (dict(dim=96), dict(R=48), dict(pages=1 << 31), dict(n=1 << 30)):
        assert call(**bad) == d.DKV_ERR_UNSUPPORTED, bad
    for bad in (dict(kn=MIS), dict(vn=MIS), dict(k=MIS), dict(v=MIS), dict(stride=257), dict(slots=ODD)):
        assert call(**bad) == d.DKV_ERR_MISALIGNED, bad
    assert call(n=0, kn=NUL, vn=NUL, slots=NUL) == d.DKV_OK


def test_binding_refuses_what_the_kernels_would_misread():
    import torch
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):  # host tensors
        d.dkv_page_release(i(2, 3), i(9), i(1), i(64))
    with pytest.raises(ValueError):  # a table of other segments
        d.dkv_page_extend(i(2), i(2), i(9), i(1), i(3, 4), 128, 2, i(3), i(2), torch.zeros(5, 2, dtype=torch.int64), i(64))
    x = torch.zeros(4, 6, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        d.dkv_paged_append(x[:, :2], x[:, 2:4], torch.zeros(4, 2, dtype=torch.int64), torch.zeros(3, 32, 64), x)


def test_paged_query_validation():
    lib = d.library()
    ws = d.dkv_paged_query_workspace_bytes(1, 32, 8, 128, 40, 40, 0)

    def call(dtype=d.DKV_BF16, B=1, Hq=32, Hkv=8, dim=128, n=40, most=40, q=A, stride=4096, off=A, pos=A, k=A, v=A, pages=9,
             R=128, ent=A, ne=A, max_e=5, scale=1.0, hint=0, out=A, w=A, w_bytes=max(ws, 1 << 40)):
        return lib.dkv_paged_query_attn(dtype, B, Hq, Hkv, dim, n, most, q, stride, off, pos, k, v, pages, R, ent, ne,
                                        max_e, scale, hint, out, w, w_bytes, NUL)

    for bad in (dict(dtype=7), dict(B=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=33), dict(n=-1), dict(most=-1), dict(pages=-1),
                dict(max_e=-1), dict(scale=float("nan")), dict(scale=3e38), dict(stride=4095), dict(stride=1 << 31),
                dict(q=NUL), dict(off=NUL), dict(pos=NUL), dict(k=NUL), dict(v=NUL), dict(ent=NUL), dict(ne=NUL),
                dict(out=NUL)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    for bad in (dict(dtype=d.DKV_F32), dict(dim=96), dict(Hq=136), dict(B=257), dict(R=96), dict(pages=1 << 31),
                dict(max_e=(1 << 23) + 1), dict(n=1 << 30, most=1 << 30), dict(n=1 << 28, most=1 << 28)):
        assert call(**bad) == d.DKV_ERR_UNSUPPORTED, bad
    for bad in (dict(q=MIS), dict(k=MIS), dict(v=MIS), dict(out=MIS), dict(ent=MIS), dict(stride=4100)):
        assert call(**bad) == d.DKV_ERR_MISALIGNED, bad
    for nothing in (dict(B=0), dict(n=0), dict(most=0)):
        assert call(q=NUL, off=NUL, pos=NUL, k=NUL, v=NUL, ent=NUL, ne=NUL, out=NUL, w=NUL, w_bytes=0, **nothing) == d.DKV_OK
    assert d.dkv_paged_query_workspace_bytes(1, 32, 8, 96, 40, 40, 0) == 0
    if ws:
        for bad in (dict(w=NUL), dict(w=MIS), dict(w_bytes=ws - 1)):
            assert call(**bad) == d.DKV_ERR_WORKSPACE, bad
