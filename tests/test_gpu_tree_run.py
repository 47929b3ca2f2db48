"""A server's loop over the paged calls, as they are used together: pages for the
drafted tokens, their plan, the cache's new rows, the attention, the accepted
path and the pages behind it, prompts first and trees after, in both formats.
Every call is compared with the oracle on the state that the calls before it left,
and the cache with the rows of the tokens that were accepted, from the beginning.

Tolerances: a row of the cache is the nearest of the format to the fp32 rounding
of its value (2^-24 of it): bf16 2^-8 of it, e4m3 2^-4 of it or half its smallest step, 2^-10
* 2^e, e the row's exponent.  Attention: as the tests of that call, fp32 sums as
random walks of 2^-24 steps with a factor of four, and 2^-20 for the
exponential and the parts of a weight."""

import numpy as np
import pytest
import torch

from oracle import page_fill as pf
from oracle import tree_cache as tc

pytestmark = pytest.mark.gpu

DEV = "cuda"
KEEP = 77.0


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


def _i32(*shape, fill=0):
    return torch.full(shape, fill, dtype=torch.int32, device=DEV)


class Server:
    """The device's buffers of B sequences over L layers, and a step of the calls."""

    def __init__(self, d, fmt, L, B, Hq, Hkv, dim, R, pages, pps, tokens, max_q, max_path, seed):
        self.d, self.fmt, self.L, self.B, self.Hq, self.Hkv, self.dim, self.R = d, fmt, L, B, Hq, Hkv, dim, R
        self.tokens, self.max_q = tokens, max_q  # of a layer
        N, S = L * B, L * B * Hkv
        self.N, self.S, self.pps, self.pages = N, S, pps, pages
        rng = np.random.default_rng(seed)
        self.free = torch.from_numpy(rng.permutation(pages).astype(np.int32)).to(DEV)
        self.n_free = _i32(1, fill=pages)
        self.table, self.len = _i32(S, pps, fill=-1), _i32(N)
        self.tok_off, self.first, self.slots = _i32(N + 1), _i32(N), torch.zeros(L * tokens, Hkv, dtype=torch.int64, device=DEV)
        self.held = _i32(N)                      # lengths with the drafted tokens
        self.entries, self.n_entries = _i32(S, pps, 4, fill=-1), _i32(S)
        self.need = torch.zeros(1, dtype=torch.int64, device=DEV)
        self.ws_extend = torch.zeros(max(16, d.dkv_page_extend_workspace_bytes(N)), dtype=torch.uint8, device=DEV)
        self.ws_release = torch.zeros(max(16, d.dkv_page_release_workspace_bytes(S, pps)), dtype=torch.uint8, device=DEV)
        self.scales = None
        if fmt == "f8":
            raw = torch.full((2, pages, R, dim), 0x7F, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
            self.scales = torch.full((pages, R, 2), 0xFF, dtype=torch.uint8, device=DEV)
        else:
            raw = torch.full((2, pages, R, dim), float("nan"), dtype=torch.bfloat16, device=DEV)
        self.k, self.v = raw[0], raw[1]
        self.freq = d.dkv_rope_freqs(d.DKV_ROPE_PLAIN, dim // 2, 10000.0)[0].to(DEV)
        # what a step is given
        self.new, self.parent = _i32(N), _i32(tokens)
        self.path, self.n_path = _i32(B, max_path), _i32(B)
        self.qkv = torch.zeros(L * tokens, Hq + 2 * Hkv, dim, dtype=torch.bfloat16, device=DEV)  # a fused projection's
        # and leaves behind
        self.pos, self.mask = _i32(tokens), torch.zeros(tokens, -(-max_q // 64), dtype=torch.int64, device=DEV)
        self.q = torch.full((L * tokens, Hq, dim), KEEP, dtype=torch.bfloat16, device=DEV)
        self.out = torch.full((L * tokens, Hq, dim), KEEP, device=DEV)
        self.keep = torch.zeros(S, pps, dtype=torch.uint8, device=DEV)
        self.hint = S // L * pps * R // 2
        ask = (d.DKV_CACHE_F8 if fmt == "f8" else d.DKV_CACHE_BF16, B, Hq, Hkv, dim, tokens, max_q, self.hint)
        self.ws = torch.full((max(16, d.dkv_paged_tree_workspace_bytes(*ask)),), 0xFF, dtype=torch.uint8, device=DEV)

    def state(self):
        return {n: t for n, t in vars(self).items() if isinstance(t, torch.Tensor) and not n.startswith("ws")}

    def draft(self, unit_new, parent, path, n_path, qkv):
        for t, x in ((self.new, unit_new), (self.parent, parent), (self.path, path), (self.n_path, n_path)):
            t.copy_(torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)))
        self.qkv.copy_(qkv)

    def extend(self):
        self.d.dkv_page_extend(self.new, self.len, self.free, self.n_free, self.table, self.R, self.Hkv, self.tok_off, self.first,
                               self.slots, self.ws_extend, new_len=self.held, entries=self.entries, n_entries=self.n_entries,
                               pages_needed=self.need)

    def attend(self, tokens):
        """tokens: rows of a layer (all of a padded batch's where there is one layer)."""
        d, B, Hq, Hkv, dim = self.d, self.B, self.Hq, self.Hkv, self.dim
        off, first = self.tok_off[:B + 1], self.first[:B]
        pos, mask, parent = self.pos[:tokens], self.mask[:tokens], self.parent[:tokens]
        d.dkv_tree_plan(off, first, self.max_q, pos, parent=parent, mask=mask)
        for l in range(self.L):
            at = slice(l * tokens, (l + 1) * tokens)
            x, segs = self.qkv[at], slice(l * B * Hkv, (l + 1) * B * Hkv)
            d.dkv_paged_store(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], self.slots[at], self.k, self.v, scales=self.scales, q=x[:, :Hq],
                              q_out=self.q[at], pos=pos, inv_freq=self.freq, rot_dim=dim // 2)
            d.dkv_paged_tree_attn(self.q[at], off, first, self.k, self.v, self.entries[segs], self.n_entries[segs], dim ** -0.5,
                                  self.out[at], self.ws, Hkv, self.max_q, mask=mask, scales=self.scales, rows_hint=self.hint)

    def accept(self):
        # a unit that was not served is left out: it keeps its length and its pages
        self.keep.fill_(1)
        self.d.dkv_paged_accept(self.first, self.path, self.n_path, self.table, self.Hkv, self.k, self.v, self.len,
                                scales=self.scales, keep=self.keep)
        self.d.dkv_page_release(self.table, self.free, self.n_free, self.ws_release, keep=self.keep)


def _trees(rng, new, tokens):
    """Parents of every drafted token and a path from a root on, for each sequence."""
    parent, paths, at = np.zeros(tokens, dtype=np.int64), [], 0
    for n in new:
        up = [int(rng.integers(max(-1, t - 4), t)) if t else -1 for t in range(max(n, 0))]
        parent[at:at + len(up)] = up
        at += len(up)
        node, line = (int(rng.integers(0, n)) if n > 0 else -1), []
        while node >= 0:
            line.append(node)
            node = up[node]
        paths.append(line[::-1][:int(rng.integers(0, len(line) + 1))] if rng.uniform() < 0.3 else line[::-1])
    return parent, paths


def _host(t):
    return t.cpu().view(torch.uint8).numpy().copy() if t.dtype is torch.float8_e4m3fn else t.cpu().float().numpy().copy() \
        if t.dtype is torch.bfloat16 else t.cpu().numpy().copy()


def _values(s):
    k, v = _host(s.k), _host(s.v)
    if s.fmt != "f8":
        return k.astype(np.float64), v.astype(np.float64)
    ex = _host(s.scales)
    return tc.row_values(k, ex[..., 0]), tc.row_values(v, ex[..., 1])


def _row_error(s, got, want):
    """Largest error of rows [..., d] in units of the tolerance."""
    size = np.abs(want)
    if s.fmt == "f8":
        _, ex = tc.quantise(want)
        half = np.maximum(size * 2.0 ** -4, (2.0 ** -10 * 2.0 ** (ex.astype(np.float64) - 127))[..., None])
    else:
        half = size * 2.0 ** -8
    return float((np.abs(got - want) / (half + size * 2.0 ** -23 + 1e-38)).max(initial=0.0))


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
@pytest.mark.parametrize("dim, Hq, Hkv, R", [(64, 8, 2, 32), (128, 6, 2, 64)])
def test_prompts_then_trees(d, fmt, dim, Hq, Hkv, R):
    L, B, tokens, max_q = 2, 3, 120, 70
    pps, pages = 8, 96
    s = Server(d, fmt, L, B, Hq, Hkv, dim, R, pages, pps, tokens, max_q, 64, 3)
    rng = np.random.default_rng([dim, 11])
    freq = s.freq.cpu().numpy()
    history = [[(np.zeros((0, Hkv, dim)), np.zeros((0, Hkv, dim))) for _ in range(B)] for _ in range(L)]
    # prompts as chains, accepted whole; then trees; one sequence waits for a step, one ends and starts anew
    plan = [[40, 3, 64], [9, 17, 1], [24, -1, 30], [1, 5, 70], [64, 2, 7], [12, 12, 12]]
    for step, new in enumerate(plan):
        T = sum(max(n, 0) for n in new)
        if step == 0:
            parent, paths = np.concatenate([np.arange(n) - 1 for n in new]), [list(range(n)) for n in new]
        else:
            parent, paths = _trees(rng, new, T)
        parent = np.concatenate([parent, np.zeros(tokens - T, np.int64)])
        path = np.zeros((B, 64), np.int64)
        for b, line in enumerate(paths):
            path[b, :len(line)] = line[:64]
        x = torch.from_numpy(rng.standard_normal((L * tokens, Hq + 2 * Hkv, dim)).astype(np.float32)).bfloat16()
        s.draft(np.tile(new, L), parent, path, [min(64, len(p)) for p in paths], x)
        before = {n: _host(t) for n, t in s.state().items()}
        s.extend()
        want = pf.page_extend(np.tile(new, L), before["len"], before["free"][:before["n_free"][0]].tolist(), before["table"], R, Hkv,
                              L * tokens, before["entries"], before["n_entries"])
        np.testing.assert_array_equal(_host(s.table), want["table"])
        np.testing.assert_array_equal(_host(s.first), want["first_pos"])
        np.testing.assert_array_equal(_host(s.slots), want["slots"])
        off, first = _host(s.tok_off)[:B + 1], _host(s.first)
        assert off[-1] == T and ((first >= 0) == (np.tile(new, L) >= 0)).all()
        slots = _host(s.slots)
        s.attend(T)
        # the plan
        pos, mask = tc.tree_plan(off, first[:B], max_q, T, parent, s.mask.shape[1])
        np.testing.assert_array_equal(_host(s.pos)[:T], pos)
        np.testing.assert_array_equal(_host(s.mask)[:T].view(np.uint64), mask)
        # the rows that were written, and no others
        k, v = _values(s)
        written = np.zeros(pages * R, dtype=bool)
        x = x.double().numpy()
        rotated = [tc.rope(x[l * T:(l + 1) * T, :Hq + Hkv], pos, freq, dim // 2) for l in range(L)]
        for l in range(L):
            at = slots[l * T:(l + 1) * T]
            written[at.reshape(-1)] = True
            assert _row_error(s, k.reshape(-1, dim)[at], rotated[l][:, Hq:]) <= 1
            assert _row_error(s, v.reshape(-1, dim)[at], x[l * T:(l + 1) * T, Hq + Hkv:]) <= 1
            got = _host(s.q)[l * T:(l + 1) * T].astype(np.float64)
            assert (np.abs(got - rotated[l][:, :Hq]) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(rotated[l][:, :Hq])).all()
        for n in ("k", "v", "scales"):
            if n in before:
                np.testing.assert_array_equal(_host(getattr(s, n)).reshape(pages * R, -1)[~written],
                                              before[n].reshape(pages * R, -1)[~written])
        # the attention
        k0, v0 = np.nan_to_num(k), np.nan_to_num(v)
        ent, n_ent, out = _host(s.entries), _host(s.n_entries), _host(s.out).astype(np.float64)
        for l in range(L):
            segs, qr = slice(l * B * Hkv, (l + 1) * B * Hkv), _host(s.q)[l * T:(l + 1) * T].astype(np.float64)
            args = (R, ent[segs], n_ent[segs], dim ** -0.5, Hkv, max_q, mask)
            want = tc.tree_attn(qr, off, first[:B], k0, v0, *args)
            size = tc.tree_attn(qr, off, first[:B], k0, np.abs(v0), *args).max(axis=2)
            big = dim ** -0.5 * np.abs(qr).max(axis=2) * np.abs(k0).sum(axis=2).max()
            tol = (4 * np.sqrt(dim) * big + 16 + 4 * np.sqrt(pps * R)) * 2.0 ** -24 * size
            err = np.abs(out[l * T:(l + 1) * T] - want).max(axis=2)
            assert (err <= tol).all(), (step, l, np.argwhere(err > tol)[:4], err.max())
        assert (out[L * T:] == before["out"][L * T:]).all()
        # the accepted path
        pools = [_host(t).reshape(pages, R, -1) for t in (s.k, s.v) + (() if s.scales is None else (s.scales,))]
        table, free = _host(s.table), _host(s.free)[:_host(s.n_free)[0]].tolist()
        s.accept()
        n_path = np.array([min(64, len(p)) for p in paths])
        want, new_len, keep = tc.accept(first, path, n_path, table, R, Hkv, pools)
        for t, y in zip((s.k, s.v, s.scales), want):
            np.testing.assert_array_equal(_host(t).reshape(pages, R, -1), y)
        held = [before["len"][n] if x is None else x for n, x in enumerate(new_len)]
        assert _host(s.len).tolist() == held
        want_table, want_free = pf.page_release(table, np.where(keep < 0, 1, keep), free, pages)
        np.testing.assert_array_equal(_host(s.table), want_table)
        assert _host(s.free)[:_host(s.n_free)[0]].tolist() == want_free
        # the cache is the accepted tokens', each at its place, through the table
        k, v = _values(s)
        for l in range(L):
            for b in range(B):
                rows = [l * T + off[b] + j for j in paths[b][:64]]
                hk, hv = history[l][b]
                if rows:
                    hk = np.concatenate([hk, x[rows, Hq:Hq + Hkv]])
                    hv = np.concatenate([hv, x[rows, Hq + Hkv:]])
                history[l][b] = hk, hv
                n = len(hk)
                assert n == held[l * B + b]
                turned, at = tc.rope(hk, np.arange(n), freq, dim // 2), np.arange(n)
                for g in range(Hkv):
                    page = _host(s.table)[(l * B + b) * Hkv + g, at // R]
                    assert _row_error(s, k[page, at % R], turned[:, g]) <= 1
                    assert _row_error(s, v[page, at % R], hv[:, g]) <= 1
        # dkv_paged_load gives the same rows
        n = held[0]
        at = torch.from_numpy(_host(s.table)[:Hkv, np.arange(n) // R].T.astype(np.int64) * R + np.arange(n)[:, None] % R).to(DEV)
        lk, lv = (torch.full((n, Hkv, dim), KEEP, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        if n:
            d.dkv_paged_load(at.contiguous(), s.k, s.v, lk, lv, scales=s.scales)
            at = at.cpu().numpy()
            np.testing.assert_array_equal(lk.cpu().double().numpy(), k.reshape(-1, dim)[at])
            np.testing.assert_array_equal(lv.cpu().double().numpy(), v.reshape(-1, dim)[at])


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
@pytest.mark.parametrize("Hq, Hkv, tokens, max_q", [(8, 2, 20, 6), (16, 2, 96, 32), (8, 1, 200, 70)])
def test_a_captured_step_replays(d, fmt, Hq, Hkv, tokens, max_q):
    """A whole step in one graph over padded batches, replayed with other trees, lengths and paths between eager work
    and synchronisations, is the eager step bit by bit; with few pages, so that some units are not served."""
    B, dim, R, pps = 3, 128, 32, 12
    make = lambda: Server(d, fmt, 1, B, Hq, Hkv, dim, R, 5 * Hkv * B, pps, tokens, max_q, 16, 5)  # noqa: E731
    eager, replayed = make(), make()
    rng = np.random.default_rng([tokens, 1])

    def step(s):
        s.extend()
        s.attend(tokens)
        s.accept()

    def draw():
        new = rng.integers(-1, min(max_q, tokens // B) + 1, size=B)
        parent, paths = _trees(rng, new, tokens)
        path = np.zeros((B, 16), np.int64)
        for b, line in enumerate(paths):
            path[b, :min(16, len(line))] = line[:16]
        x = torch.from_numpy(rng.standard_normal((tokens, Hq + 2 * Hkv, dim)).astype(np.float32)).bfloat16()
        return new, parent, path, [min(16, len(p)) for p in paths], x

    # warm up on buffers of its own, then record
    side = make()
    side.draft(*draw())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(side)
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed)
    for trial in range(8):
        given = draw()
        for s in (eager, replayed):
            s.draft(*given)
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        for (name, a), b in zip(eager.state().items(), replayed.state().values()):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (trial, name)
        # rows behind the last sequence are nobody's
        end = int(eager.tok_off[B])
        assert (eager.pos[end:] == -1).all() and (trial > 0 or (eager.out[end:] == KEEP).all())
        assert torch.isfinite(eager.out).all()


@pytest.mark.parametrize("fmt", ["f8", "bf16"])
def test_two_streams_at_once(d, fmt):
    """Two servers' steps side by side, each on its own stream and buffers, are the steps alone."""
    args = (fmt, 1, 2, 8, 2, 64, 32, 60, 9, 40, 20, 16)
    rng = np.random.default_rng(9)
    given = []
    for _ in range(2):
        new = rng.integers(1, 21, size=2)
        parent, paths = _trees(rng, new, 40)
        path = np.zeros((2, 16), np.int64)
        for b, line in enumerate(paths):
            path[b, :min(16, len(line))] = line[:16]
        given.append((new, parent, path, [min(16, len(p)) for p in paths],
                      torch.from_numpy(rng.standard_normal((40, 12, 64)).astype(np.float32)).bfloat16()))
    alone, both = ([Server(d, *args, seed) for seed in (1, 2)] for _ in range(2))
    for servers in (alone, both):
        for s, g in zip(servers, given):
            s.draft(*g)
    torch.cuda.synchronize()
    for s in alone:
        s.extend(), s.attend(40), s.accept()
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for call in (lambda s: s.extend(), lambda s: s.attend(40), lambda s: s.accept()):
        for s, stream in zip(both, streams):
            with torch.cuda.stream(stream):
                call(s)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for (name, x), y in zip(a.state().items(), b.state().values()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), name
