"""Rotary positions, quantised rows and drafted trees, on the host: the oracle's
results worked out by hand or by another route, the frequencies, and the entry
points' refusals (no call passes validation, so nothing reaches a GPU)."""

import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_32663_amd as d
from oracle import page_fill as pf
from oracle import tree_cache as tc

A = ctypes.c_void_p(0x10000)    # fake 16-byte-aligned device address
MIS = ctypes.c_void_p(0x10008)  # 8-byte-aligned only
ODD = ctypes.c_void_p(0x10002)
NUL = None
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---------------------------------------------------------------------------
# the oracle
# ---------------------------------------------------------------------------

def test_rope_is_a_rotation_of_complex_numbers():
    rng = np.random.default_rng(1)
    x, pos, f = rng.standard_normal((5, 3, 24)), np.array([0, 1, 7, -1, 100000]), rng.uniform(0, 1, 9).astype(np.float32)
    half, pairs = (tc.rope(x, pos, f, 18, i, 1.5) for i in (False, True))
    for t in (0, 1, 2, 4):
        turn = 1.5 * np.exp(1j * float(pos[t]) * f.astype(np.float64))
        z = (x[t, :, :9] + 1j * x[t, :, 9:18]) * turn
        np.testing.assert_allclose(half[t, :, :18], np.concatenate([z.real, z.imag], axis=1), atol=1e-12)
        z = (x[t, :, 0:18:2] + 1j * x[t, :, 1:18:2]) * turn
        np.testing.assert_allclose(pairs[t, :, :18], np.stack([z.real, z.imag], axis=2).reshape(3, 18), atol=1e-12)
    for y in (half, pairs):
        np.testing.assert_array_equal(y[..., 18:], x[..., 18:])
        np.testing.assert_array_equal(y[3], x[3])


def test_codes_are_torchs_e4m3():
    code = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(tc.codes_to_values(code.numpy()), code.view(torch.float8_e4m3fn).double().numpy())
    x = torch.cat([torch.linspace(-448, 448, 20001), torch.linspace(-0.1, 0.1, 20001)]).double()
    x = torch.cat([x, torch.from_numpy(tc._BORDERS), -torch.from_numpy(tc._BORDERS)])
    rows = torch.stack([x, torch.full_like(x, 448.0)], dim=-1).numpy()  # the second keeps the exponent at 0
    codes, ex = tc.quantise(rows)
    assert (ex == 127).all()
    np.testing.assert_array_equal(tc.codes_to_values(codes[:, 0]), x.float().to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("most, e", [(448.0, 0), (448.0000001, 1), (1.75, -8), (1.7500001, -7), (1.0, -8), (2.0, -7),
                                     (0.0, -60), (1e-38, -60), (3.0e38, 120), (1.75 * 2.0 ** -51, -59),
                                     (1.75 * 2.0 ** -52, -60), (2.0 ** -52, -60)])
def test_exponent_of_a_row(most, e):
    codes, ex = tc.quantise(np.array([[most, -most / 3, 0.0]]))
    assert int(ex[0]) - 127 == e
    v = tc.row_values(codes, ex)[0]
    if most >= 2.0 ** -52:
        assert abs(v[0] - most) <= most * 2.0 ** -4


def test_quantise_extremes():
    big = float(torch.finfo(torch.bfloat16).max)
    codes, ex = tc.quantise(np.array([[big, np.nan, np.inf, -np.inf, 1.0]]))
    v = tc.row_values(codes, ex)[0]
    assert v[0] == 240.0 * 2.0 ** 120 and np.isnan(v[1:4]).all() and v[4] == 0.0
    codes, ex = tc.quantise(np.array([[np.inf, 3.0]]))  # an infinity does not set the exponent
    assert tc.row_values(codes, ex)[0, 1] == 3.0
    assert torch.tensor(v[:1]).bfloat16().isfinite().all()


def test_plan_by_hand():
    #      0        chunk 1: a chain of two; padded rows
    #    1   2      -> 3 under 1, 4 under 3, 5 a second root
    parent = [-1, 0, 0, 1, 3, -1, 7, 0]
    pos, mask = tc.tree_plan([0, 6, 8], [10, 4], 6, 9, parent, 1)
    np.testing.assert_array_equal(pos, [10, 11, 11, 12, 13, 10, 4, 5, -1])
    np.testing.assert_array_equal(mask[:, 0], [1, 3, 5, 11, 27, 32, 1, 3, 0])
    pos, mask = tc.tree_plan([0, 3], [0], 3, 3, None, 1)
    np.testing.assert_array_equal(mask[:, 0], [1, 3, 7])


def test_accept_by_hand():
    pool = np.arange(4 * 2).reshape(4, 2, 1)  # four pages of two rows (two, though the library has none so small)
    table = np.array([[3, 0, 2, -1]])
    (moved,), new_len, keep = tc.accept([1], np.array([[0, 2, 3, 3]]), [4], table, 2, 1, [pool])
    # positions 1 .. 4 are rows 7, 0, 1, 4; the path's tokens 0, 2, 3 are at 1, 3, 4 and go to 1, 2, 3
    assert new_len == [4] and keep.tolist() == [[1, 1, 0, 0]]
    assert moved.reshape(-1).tolist() == [1, 4, 2, 3, 4, 5, 6, 7]


def test_tree_attention_without_a_mask_is_the_chunks():
    """Chains give the same as the causal chunk, with the mask of a chain and without one."""
    rng = np.random.default_rng(2)
    R, Hkv, G, dim, held, new = 32, 2, 2, 64, [40, 0, 7], [3, 5, 1]
    f = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    table = rng.permutation(6 * 3).reshape(6, 3)
    k, v, q = f(18, R, dim), f(18, R, dim), f(9, Hkv * G, dim)
    total = np.repeat(np.array(held) + new, Hkv)
    ent = [[(table[s, p], p, 0, min(R, total[s] - p * R)) for p in range(-(-total[s] // R))] + [(0, 0, 0, 0)] * 2 for s in range(6)]
    ent = np.array([x[:2] for x in ent])
    n_ent = -(-total // R)
    off = [0, 3, 8, 9]
    import oracle as o
    want = pf.chunk_attn(q, off, held, k, v, ent, n_ent, 0.2, Hkv, o.F32, 5)
    _, mask = tc.tree_plan(off, held, 5, 9, None, 1)
    for m in (None, mask):
        got = tc.tree_attn(q.astype(np.float64), off, held, k.astype(np.float64), v.astype(np.float64), R, ent, n_ent, 0.2,
                           Hkv, 5, m)
        np.testing.assert_allclose(got, want, rtol=1e-12, atol=1e-13)
    mask[4] = 0  # sequence 1 holds nothing: its token 1 now sees nothing
    got = tc.tree_attn(q.astype(np.float64), off, held, k.astype(np.float64), v.astype(np.float64), R, ent, n_ent, 0.2,
                       Hkv, 5, mask)
    assert (got[4] == 0).all() and np.isfinite(got).all()


# ---------------------------------------------------------------------------
# frequencies
# ---------------------------------------------------------------------------

def test_plain_and_linear_frequencies():
    f, m = d.dkv_rope_freqs(d.DKV_ROPE_PLAIN, 128, 10000.0)
    want = torch.tensor([10000.0 ** (-2 * i / 128) for i in range(64)], dtype=torch.float64)
    assert m == 1.0 and torch.equal(f, want.float())
    g, m = d.dkv_rope_freqs(d.DKV_ROPE_LINEAR, 128, 10000.0, 4.0)
    assert m == 1.0 and torch.equal(g, (want / 4).float())


def test_stretched_bases_ends():
    f, m = d.dkv_rope_freqs(d.DKV_ROPE_BASE, 64, 10000.0, 8.0)
    p, _ = d.dkv_rope_freqs(d.DKV_ROPE_PLAIN, 64, 10000.0)
    assert m == 1.0 and f[0] == 1.0 and abs(f[-1] / p[-1] * 8 - 1) < 1e-6


@pytest.mark.parametrize("kind", [d.DKV_ROPE_WAVE, d.DKV_ROPE_RAMP])
def test_stretched_by_bands(kind):
    """Pairs that turn often stay, slow ones are divided, and between them each is between both."""
    f, m = d.dkv_rope_freqs(kind, 128, 500000.0, 8.0, 8192.0, 1.0, 4.0)
    p, _ = d.dkv_rope_freqs(d.DKV_ROPE_PLAIN, 128, 500000.0)
    turns = 8192.0 * p.double() / (2 * math.pi)
    assert torch.equal(f[turns >= 8.0], p[turns >= 8.0])
    slow = turns < 0.5
    assert torch.equal(f[slow], (p.double() / 8).float()[slow]) or torch.allclose(f[slow], p[slow] / 8, rtol=2.0 ** -23)
    assert ((f <= p) & (f >= p / 8 * (1 - 2.0 ** -22))).all()
    i = int(((turns > 1.0) & (turns < 4.0)).nonzero()[0])
    if kind == d.DKV_ROPE_WAVE:
        keep = (turns[i] - 1.0) / 3.0
        assert m == 1.0
    else:
        at = lambda t: 128 * math.log(8192.0 / (2 * math.pi * t)) / (2 * math.log(500000.0))  # noqa: E731
        keep = 1 - (i - math.floor(at(4.0))) / (math.ceil(at(1.0)) - math.floor(at(4.0)))
        assert abs(m - (0.1 * math.log(8.0) + 1.0)) < 1e-6
    want = keep * p[i].double() + (1 - keep) * p[i].double() / 8
    assert abs(f[i].double() / want - 1) < 2.0 ** -22


def test_frequency_refusals():
    lib = d.library()
    f, m = torch.empty(64), ctypes.c_float()

    def call(kind=3, rot=128, base=1e4, factor=2.0, length=4096.0, low=1.0, high=4.0, out=f.data_ptr(), ms=ctypes.byref(m)):
        return lib.dkv_rope_freqs(kind, rot, base, factor, length, low, high, out, ms)

    assert call() == d.DKV_OK
    nan = float("nan")
    for bad in (dict(kind=5), dict(kind=-1), dict(rot=0), dict(rot=3), dict(rot=-2), dict(base=1.0), dict(base=nan),
                dict(factor=0.5), dict(factor=nan), dict(length=0.0), dict(length=nan), dict(low=0.0), dict(high=1.0),
                dict(low=nan), dict(high=float("inf")), dict(out=NUL), dict(ms=NUL), dict(kind=2, rot=2)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    with pytest.raises(d.DkvError):
        d.dkv_rope_freqs(d.DKV_ROPE_PLAIN, 0, 1e4)


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------

def test_rope_validation():
    lib = d.library()

    def call(dtype=d.DKV_BF16, n=4, heads=6, dim=128, x=A, xs=768, pos=A, f=A, rot=128, inter=0, ms=1.0, out=A, os=768):
        return lib.dkv_rope(dtype, n, heads, dim, x, xs, pos, f, rot, inter, ms, out, os, NUL)

    for bad in (dict(dtype=2), dict(n=-1), dict(heads=0), dict(rot=0), dict(rot=-2), dict(rot=7), dict(rot=130),
                dict(ms=float("nan")), dict(xs=767), dict(os=767), dict(xs=1 << 31), dict(x=NUL), dict(pos=NUL),
                dict(f=NUL), dict(out=NUL)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    for bad in (dict(dim=132, xs=792, os=792), dict(dim=264, xs=1584, os=1584), dict(n=1 << 22)):
        assert call(**bad) == d.DKV_ERR_UNSUPPORTED, bad
    for bad in (dict(x=MIS), dict(out=MIS), dict(xs=772), dict(os=772)):
        assert call(**bad) == d.DKV_ERR_MISALIGNED, bad
    assert call(n=0, x=NUL, pos=NUL, f=NUL, out=NUL) == d.DKV_OK


def test_store_validation():
    lib = d.library()

    def call(fmt=d.DKV_CACHE_F8, n=4, Hq=4, Hkv=2, dim=128, q=A, qs=512, kn=A, vn=A, kvs=256, pos=A, f=A, rot=128, inter=0,
             ms=1.0, qo=A, qos=512, slots=A, k=A, v=A, ex=A, pages=9, R=128):
        return lib.dkv_paged_store(fmt, n, Hq, Hkv, dim, q, qs, kn, vn, kvs, pos, f, rot, inter, ms, qo, qos, slots, k, v,
                                   ex, pages, R, NUL)

    for bad in (dict(fmt=2), dict(fmt=-1), dict(n=-1), dict(Hq=-1), dict(Hkv=0), dict(pages=-1), dict(rot=-2), dict(rot=3),
                dict(rot=130), dict(ms=float("inf")), dict(kvs=255), dict(qs=511), dict(qos=511), dict(kvs=1 << 31),
                dict(q=NUL), dict(qo=NUL), dict(kn=NUL), dict(vn=NUL), dict(pos=NUL), dict(f=NUL), dict(slots=NUL),
                dict(k=NUL), dict(v=NUL), dict(ex=NUL)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    for bad in (dict(dim=96, rot=96), dict(R=48), dict(R=16), dict(pages=1 << 31), dict(n=1 << 22), dict(Hq=1 << 20, qs=1 << 30, qos=1 << 30)):
        assert call(**bad) == d.DKV_ERR_UNSUPPORTED, bad
    for bad in (dict(q=MIS), dict(qo=MIS), dict(kn=MIS), dict(vn=MIS), dict(k=MIS), dict(v=MIS), dict(slots=ODD),
                dict(ex=ODD), dict(qs=516), dict(qos=516), dict(kvs=260)):
        assert call(**bad) == d.DKV_ERR_MISALIGNED, bad
    assert call(n=0, q=NUL, qo=NUL, kn=NUL, vn=NUL, slots=NUL) == d.DKV_OK


def test_load_validation():
    lib = d.library()

    def call(fmt=d.DKV_CACHE_F8, n=4, Hkv=2, dim=128, k=A, v=A, ex=A, pages=9, R=128, slots=A, ko=A, vo=A, stride=256):
        return lib.dkv_paged_load(fmt, n, Hkv, dim, k, v, ex, pages, R, slots, ko, vo, stride, NUL)

    for bad in (dict(fmt=7), dict(n=-1), dict(Hkv=0), dict(pages=-1), dict(stride=255), dict(stride=1 << 31), dict(k=NUL),
                dict(v=NUL), dict(ex=NUL), dict(slots=NUL), dict(ko=NUL), dict(vo=NUL)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    for bad in (dict(dim=256, stride=512), dict(R=100), dict(pages=1 << 31), dict(n=1 << 28)):
        assert call(**bad) == d.DKV_ERR_UNSUPPORTED, bad
    for bad in (dict(k=MIS), dict(v=MIS), dict(ko=MIS), dict(vo=MIS), dict(slots=ODD), dict(ex=ODD), dict(stride=257)):
        assert call(**bad) == d.DKV_ERR_MISALIGNED, bad
    assert call(n=0, slots=NUL) == d.DKV_OK and call(pages=0, k=NUL, v=NUL) == d.DKV_OK


def test_plan_validation():
    lib = d.library()

    def call(B=2, n=80, most=70, off=A, first=A, parent=A, pos=A, mask=A, words=2):
        return lib.dkv_tree_plan(B, n, most, off, first, parent, pos, mask, words, NUL)

    for bad in (dict(B=-1), dict(n=-1), dict(most=-1), dict(words=-1), dict(words=1), dict(off=NUL), dict(first=NUL),
                dict(pos=NUL)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    for bad in (dict(n=2000, most=1025, words=32), dict(B=2049)):
        assert call(**bad) == d.DKV_ERR_UNSUPPORTED, bad
    assert call(mask=ODD) == d.DKV_ERR_MISALIGNED
    assert call(n=0, off=NUL, pos=NUL) == d.DKV_OK


def test_accept_validation():
    lib = d.library()

    def call(fmt=d.DKV_CACHE_F8, N=4, B=2, Hkv=2, dim=128, first=A, path=A, n_path=A, most=8, table=A, pps=5, R=128, k=A, v=A,
             ex=A, pages=9, new_len=ctypes.c_void_p(0x20000), keep=A):
        return lib.dkv_paged_accept(fmt, N, B, Hkv, dim, first, path, n_path, most, table, pps, R, k, v, ex, pages, new_len,
                                    keep, NUL)

    for bad in (dict(fmt=3), dict(N=-1), dict(B=-1), dict(B=0), dict(B=3), dict(Hkv=0), dict(most=-1), dict(pps=-1),
                dict(pages=-1), dict(first=NUL), dict(path=NUL), dict(n_path=NUL), dict(table=NUL), dict(new_len=NUL), dict(new_len=A),
                dict(k=NUL), dict(v=NUL), dict(ex=NUL)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    for bad in (dict(dim=32), dict(R=33), dict(most=65), dict(N=32768, B=2), dict(pages=1 << 31)):
        assert call(**bad) == d.DKV_ERR_UNSUPPORTED, bad
    for bad in (dict(k=MIS), dict(v=MIS), dict(ex=ODD)):
        assert call(**bad) == d.DKV_ERR_MISALIGNED, bad
    assert call(N=0, first=NUL, path=NUL, n_path=NUL, table=NUL, new_len=NUL) == d.DKV_OK


def test_tree_attention_validation():
    lib = d.library()

    def call(fmt=d.DKV_CACHE_F8, B=2, Hq=8, Hkv=2, dim=128, n=9, most=5, q=A, qs=1024, off=A, first=A, mask=A, words=1, k=A,
             v=A, ex=A, pages=9, R=128, ent=A, n_ent=A, max_ent=4, scale=0.1, hint=1000, out=A, ws=A, ws_bytes=1 << 30):
        return lib.dkv_paged_tree_attn(fmt, B, Hq, Hkv, dim, n, most, q, qs, off, first, mask, words, k, v, ex, pages, R, ent,
                                       n_ent, max_ent, scale, hint, out, ws, ws_bytes, NUL)

    for bad in (dict(fmt=2), dict(fmt=-1), dict(B=-1), dict(Hkv=0), dict(Hq=9), dict(n=-1), dict(most=-1), dict(words=-1),
                dict(pages=-1), dict(max_ent=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(qs=1023),
                dict(qs=1 << 31), dict(q=NUL), dict(off=NUL), dict(first=NUL), dict(k=NUL), dict(v=NUL), dict(ex=NUL),
                dict(ent=NUL), dict(n_ent=NUL), dict(out=NUL)):
        assert call(**bad) == d.DKV_ERR_INVALID_ARG, bad
    for bad in (dict(dim=96), dict(Hq=34, qs=34 * 128), dict(R=48), dict(R=16), dict(pages=1 << 31), dict(B=1025),
                dict(max_ent=1 << 24), dict(words=(1 << 20) + 1)):
        assert call(**bad) == d.DKV_ERR_UNSUPPORTED, bad
    for bad in (dict(q=MIS), dict(k=MIS), dict(v=MIS), dict(ex=MIS), dict(ent=MIS), dict(out=MIS), dict(qs=1028),
                dict(mask=ODD)):
        assert call(**bad) == d.DKV_ERR_MISALIGNED, bad
    big = dict(n=900, most=512, hint=1 << 20)
    need = lib.dkv_paged_tree_workspace_bytes(d.DKV_CACHE_F8, 2, 8, 2, 128, 900, 512, 1 << 20)
    assert need > 0
    for bad in (dict(ws=NUL), dict(ws=MIS), dict(ws_bytes=need - 1)):
        assert call(**big, **bad) == d.DKV_ERR_WORKSPACE, bad
    for empty in (dict(B=0), dict(n=0), dict(most=0)):
        assert call(**empty, q=NUL, out=NUL, off=NUL) == d.DKV_OK
    for bad in ((2, 2, 8, 2, 128, 9, 5, 0), (1, -1, 8, 2, 128, 9, 5, 0), (1, 2, 8, 3, 128, 9, 5, 0), (1, 2, 8, 2, 80, 9, 5, 0)):
        assert lib.dkv_paged_tree_workspace_bytes(*bad) == 0
    assert call(fmt=d.DKV_CACHE_BF16, ex=NUL, q=NUL) == d.DKV_ERR_INVALID_ARG  # no exponents there: q is what is missing


TREE_ROUTE = r"""
#include "dkv_query.hpp"
#include <cstdio>
int main() {
  long long nseg, rows, hint;
  while (std::scanf("%lld %lld %lld", &nseg, &rows, &hint) == 3)
    std::printf("%d\n", dkv::paged_f8_takes_short(nseg, rows, hint) ? 1 : 0);
}
"""


def test_quantised_blocks_take_the_faster_kernel(tmp_path):
    """The route over a quantised cache at sizes where the two kernels' times are 10% and more apart on an MI355X,
    at the rule's edges, and without a hint."""
    cxx, rocm = shutil.which("g++"), "/opt/rocm/include"
    if cxx is None or not os.path.isdir(rocm):
        pytest.skip("no host compiler or HIP headers")
    src, exe = tmp_path / "route.cpp", tmp_path / "route"
    src.write_text(TREE_ROUTE)
    subprocess.run([cxx, "-std=c++17", "-D__HIP_PLATFORM_AMD__", f"-I{rocm}",
                    f"-I{os.path.join(ROOT, 'paper_2609_32663_amd', 'csrc')}", str(src), "-o", str(exe)], check=True)
    # (segments, query rows, keys per segment, short kernel)
    sizes = [(256, 8, 8000, 1), (8, 64, 32000, 1), (2048, 64, 0, 1), (128, 64, 2000, 0),
             (128, 32, 2000, 1), (128, 64, 300, 1), (128, 64, 16000, 1), (64, 64, 4000, 1), (256, 33, 1000, 1), (65, 33, 8065, 0),
             (65, 33, 8066, 1), (128, 40, 0, 1), (8, 96, 2000, 1), (8, 96, 32000, 1), (32, 96, 2000, 1),
             (32, 96, 8000, 0), (128, 96, 300, 1), (128, 128, 2000, 0), (128, 96, 32000, 0), (16, 65, 1 << 15, 0),
             (16, 65, (1 << 15) - 1, 1), (17, 128, 3855, 1), (17, 128, 3856, 0), (16, 128, 0, 1), (17, 128, 0, 0),
             (8, 192, 300, 0), (8, 192, 2000, 1), (8, 192, 32000, 0), (32, 192, 2000, 0), (16, 256, 8192, 1),
             (16, 256, 8193, 0), (8, 257, 2000, 0), (16, 129, 0, 0)]
    out = subprocess.run([str(exe)], input="\n".join(f"{n} {r} {n * k}" for n, r, k, _ in sizes), check=True,
                         capture_output=True, text=True).stdout.split()
    assert [int(x) for x in out] == [w for *_, w in sizes]


def test_binding_refuses_what_the_kernels_would_misread():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    x, f = torch.zeros(4, 6, 64, dtype=torch.bfloat16), torch.zeros(32)
    pool, slots = torch.zeros(3, 32, 64, dtype=torch.bfloat16), torch.zeros(4, 2, dtype=torch.int64)
    for call in (lambda: d.dkv_rope(x, i(4), f, 64, x),                                  # host tensors
                 lambda: d.dkv_tree_plan(i(3), i(2), 4, i(4)),
                 lambda: d.dkv_paged_store(x[:, :2], x[:, 2:4], slots, pool, pool),
                 lambda: d.dkv_paged_load(slots, pool, pool, x[:, :2], x[:, 2:4]),
                 lambda: d.dkv_paged_accept(i(2), i(2, 8), i(2), i(5, 4), 2, pool, pool, i(2))):  # a table of others
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        d.dkv_paged_load(slots, pool.float(), pool.float(), x[:, :2], x[:, 2:4])
