"""The calls of rotation, 8-bit rows and drafted trees at the edges of their arguments: another device, bounds beyond
32 bits, lists that name slots outside their pages, prompts whose query tiles stay whole."""

import numpy as np
import pytest
import torch

from test_gpu_tree_attn import DEV, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


def _calls(d):
    """Each of the calls on small tensors, as a function of its stream."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    slots, freq = torch.zeros((4, 2), dtype=torch.int64, device=DEV), torch.ones(32, device=DEV)
    pool, x = (torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in ((3, 32, 64), (4, 2, 64)))
    b = Batch(np.random.default_rng(1), "f8", [40], [3], 2, 4, 64, 32)
    return [lambda s: d.dkv_rope(x, i32(4), freq, 64, x.clone(), stream=s),
            lambda s: d.dkv_tree_plan(i32(3), i32(2), 4, i32(4), stream=s),
            lambda s: d.dkv_paged_store(x, x, slots, pool, pool, stream=s),
            lambda s: d.dkv_paged_load(slots, pool, pool, x.clone(), x.clone(), stream=s),
            lambda s: d.dkv_paged_accept(i32(2), i32(1, 8), i32(1), i32(4, 3), 2, pool, pool, i32(2), stream=s),
            lambda s: b.run(d, stream=s)]


class _StreamOf:
    def __init__(self, device_index):
        self.device_index, self.cuda_stream = device_index, 0


@pytest.mark.parametrize("call", range(6))
def test_another_device_is_refused(d, call, monkeypatch):
    f = _calls(d)[call]
    f(None)
    f(torch.cuda.current_stream())
    with pytest.raises(ValueError, match="current device"):
        f(_StreamOf(torch.cuda.current_device() + 1))
    monkeypatch.setattr(d.binding, "_current_device", lambda: torch.cuda.current_device() + 1)
    with pytest.raises(ValueError, match="current device"):
        f(None)
    torch.cuda.synchronize()


def test_tensors_of_other_types_and_shapes_are_refused(d):
    b = Batch(np.random.default_rng(1), "f8", [40], [3], 2, 4, 64, 32)
    b.run(d)
    off, first, k, v, ent, n_ent = b.dev
    out, ws = torch.zeros(3, 8, 64, device=DEV), torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)

    def call(q=b.q_dev, off=off, first=first, k=k, v=v, ent=ent, n_ent=n_ent, out=out, mask=b.mask_dev, scales=b.scales):
        d.dkv_paged_tree_attn(q, off, first, k, v, ent, n_ent, 0.1, out, ws, 2, 3, mask=mask, scales=scales)

    call()
    for bad in (dict(q=b.q_dev.float()), dict(q=b.q_dev.transpose(0, 1)), dict(off=off.long()), dict(off=off[:1]),
                dict(first=first.long()), dict(v=v[:-1]), dict(v=v.view(torch.uint8)), dict(ent=ent[:1]), dict(n_ent=n_ent[:1]),
                dict(out=out.half()), dict(out=out[:2]), dict(mask=b.mask_dev[:2]), dict(mask=b.mask_dev.int()), dict(scales=None),
                dict(scales=b.scales[:, :16].contiguous()), dict(scales=b.scales.int()), dict(q=b.q_dev.cpu())):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(TypeError):
        call(k=k.view(torch.uint8), v=v.view(torch.uint8))
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
def test_a_longest_chunk_beyond_int32_is_all_tokens(d, fmt):
    x = Batch(np.random.default_rng(2), fmt, [300, 90], [80, 3], 2, 4, 64, 32, mask=None)
    want = x.run(d)
    x.max_q = 1 << 32
    assert torch.equal(x.run(d), want)


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
@pytest.mark.parametrize("R", [32, 64, 256, 1024])
@pytest.mark.parametrize("new", [[6, 9], [80, 140]])
def test_entries_whose_slots_end_below_zero(d, fmt, new, R):
    """An end far below zero names no slot; nor do a first slot and an end at the largest int32."""
    x = Batch(np.random.default_rng([R, new[0]]), fmt, [8 * R, 7 * R], new, 2, 4, 64, R)
    least, most = -2 ** 31, 2 ** 31 - 1
    for s in range(4):
        x.entries[s, 1, 2:] = (0, least)
        x.entries[s, 2, 2:] = (0, least + 31)
        x.entries[s, 3, 2:] = (0, least + R - 32)
        x.entries[s, 4, 2:] = (0, most)
        x.entries[s, 5, 2:] = (most, most)
    x.check(d)


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("masked", [False, True])
def test_prompts_whose_tiles_stay_whole(d, fmt, dim, masked):
    """Eight prompts of 1,500 tokens: the plan deals whole units (its third word), over both formats; against float64."""
    Hkv, G, R, B, n = 8, 4, 128, 8, 1500
    gen = torch.Generator(device=DEV).manual_seed(dim)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    i32 = lambda x: torch.as_tensor(np.asarray(x), device=DEV).to(torch.int32)  # noqa: E731
    per = -(-n // R)
    pages, tokens = B * Hkv * per, B * n
    table = torch.randperm(pages, generator=gen, device=DEV).view(B * Hkv, per)
    entries = torch.zeros((B * Hkv, per, 4), dtype=torch.int32, device=DEV)
    entries[..., 0] = table
    entries[..., 1] = torch.arange(per, device=DEV)
    entries[..., 3] = (n - entries[..., 1] * R).clamp(0, R)
    scales = None
    if fmt == "f8":
        pools = [(100 * rand(pages, R, dim)).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2)]
        scales = torch.randint(117, 123, (pages, R, 2), generator=gen, device=DEV).to(torch.uint8)
        values = [p.double() * torch.exp2(scales[..., i:i + 1].double() - 127) for i, p in enumerate(pools)]
    else:
        pools = [rand(pages, R, dim).bfloat16() for _ in range(2)]
        values = [p.double() for p in pools]
    q = rand(tokens, Hkv * G, dim).bfloat16()
    off, first = i32(np.arange(B + 1) * n), i32([0] * B)
    hint = B * Hkv * per * R
    code = d.DKV_CACHE_F8 if fmt == "f8" else d.DKV_CACHE_BF16
    ws = torch.full((d.dkv_paged_tree_workspace_bytes(code, B, Hkv * G, Hkv, dim, tokens, n, hint),), 0xFF, dtype=torch.uint8,
                    device=DEV)
    mask = None
    if masked:
        mask = torch.zeros(tokens, -(-n // 64), dtype=torch.int64, device=DEV)
        d.dkv_tree_plan(off, first, n, torch.empty(tokens, dtype=torch.int32, device=DEV), mask=mask)
    out = torch.empty((tokens, Hkv * G, dim), device=DEV)
    d.dkv_paged_tree_attn(q, off, first, *pools, entries, i32([per] * (B * Hkv)), dim ** -0.5, out, ws, Hkv, n, mask=mask,
                          scales=scales, rows_hint=hint)
    assert int(ws[8:12].view(torch.int32)) == 1
    hide = torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1)
    for s in range(0, B * Hkv, 5):
        b, g = divmod(s, Hkv)
        k, v = (x[table[s]].view(per * R, dim)[:n] for x in values)
        qs = q[b * n:(b + 1) * n, g * G:(g + 1) * G].double()
        big = dim ** -0.5 * qs.abs().amax(2) * k.abs().sum(1).max()
        for h in range(G):
            p = (qs[:, h] @ k.T * dim ** -0.5).masked_fill(hide, -float("inf")).softmax(1)
            err = (out[b * n:(b + 1) * n, g * G + h].double() - p @ v).abs().amax(1)
            tol = (4 * dim ** 0.5 * big[:, h] + 16 + 4 * n ** 0.5) * 2.0 ** -24 * (p @ v.abs()).amax(1)
            assert (err <= tol).all(), (s, h, float((err / tol).max()))


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("gaps", [False, True])
def test_ranges_of_more_runs_than_a_table_holds(d, fmt, dim, gaps):
    """32 sequences of 70,000 positions, 96 rows for each of 8 heads: a workgroup walks a whole segment, 2,188 runs of 32
    rows, whose table is filled twice; whole pages, and pages of which a part is kept.  Pages are shared."""
    Hkv, G, R, B, n, held, pool = 8, 4, 128, 32, 24, 70000, 300
    gen = torch.Generator(device=DEV).manual_seed(dim)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    i32 = lambda x: torch.as_tensor(np.asarray(x), device=DEV).to(torch.int32)  # noqa: E731
    T = held + n
    per, tokens = -(-T // R), B * n
    entries = torch.zeros((B * Hkv, per, 4), dtype=torch.int32, device=DEV)
    entries[..., 0] = torch.randint(pool, entries.shape[:2], generator=gen, device=DEV)
    entries[..., 1] = torch.arange(per, device=DEV)
    entries[..., 3] = (T - entries[..., 1] * R).clamp(0, R)
    if gaps:
        entries[:, :-2, 2] = torch.randint(0, R, (B * Hkv, per - 2), generator=gen, device=DEV).to(torch.int32)
    scales = None
    if fmt == "f8":
        pools = [(100 * rand(pool, R, dim)).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2)]
        scales = torch.randint(117, 123, (pool, R, 2), generator=gen, device=DEV).to(torch.uint8)
        values = [p.double() * torch.exp2(scales[..., i:i + 1].double() - 127) for i, p in enumerate(pools)]
    else:
        pools = [rand(pool, R, dim).bfloat16() for _ in range(2)]
        values = [p.double() for p in pools]
    q = rand(tokens, Hkv * G, dim).bfloat16()
    off, first = i32(np.arange(B + 1) * n), i32([held] * B)
    code, hint = d.DKV_CACHE_F8 if fmt == "f8" else d.DKV_CACHE_BF16, B * Hkv * per * R
    ws = torch.full((d.dkv_paged_tree_workspace_bytes(code, B, Hkv * G, Hkv, dim, tokens, n, hint),), 0xFF, dtype=torch.uint8,
                    device=DEV)
    # a tree: token t continues t - 3
    pos, mask = torch.empty(tokens, dtype=torch.int32, device=DEV), torch.zeros(tokens, 1, dtype=torch.int64, device=DEV)
    d.dkv_tree_plan(off, first, n, pos, parent=i32(np.tile(np.arange(n) - 3, B)), mask=mask)
    out = torch.empty((tokens, Hkv * G, dim), device=DEV)
    d.dkv_paged_tree_attn(q, off, first, *pools, entries, i32([per] * (B * Hkv)), dim ** -0.5, out, ws, Hkv, n, mask=mask,
                          scales=scales, rows_hint=hint)
    slot, at = torch.arange(R, device=DEV), torch.arange(n, device=DEV)
    sees = (at[:, None] - at[None] >= 0) & ((at[:, None] - at[None]) % 3 == 0)
    for s in range(0, B * Hkv, 51):
        b, g = divmod(s, Hkv)
        e = entries[s].long()
        kept = ((slot >= e[:, 2:3]) & (slot < e[:, 3:4])).view(-1)
        where = torch.arange(per * R, device=DEV)[kept]
        k, v = (x[e[:, 0]].view(per * R, dim)[kept] for x in values)
        ok = torch.ones(n, len(where), dtype=torch.bool, device=DEV)
        new = where >= held
        ok[:, new] = sees[:, where[new] - held]
        qs = q[b * n:(b + 1) * n, g * G:(g + 1) * G].double()
        big = dim ** -0.5 * qs.abs().amax(2) * k.abs().sum(1).max()
        for h in range(G):
            p = (qs[:, h] @ k.T * dim ** -0.5).masked_fill(~ok, -float("inf")).softmax(1)
            err = (out[b * n:(b + 1) * n, g * G + h].double() - p @ v).abs().amax(1)
            tol = (4 * dim ** 0.5 * big[:, h] + 16 + 4 * T ** 0.5) * 2.0 ** -24 * (p @ v.abs()).amax(1)
            assert (err <= tol).all(), (s, h, float((err / tol).max()))
