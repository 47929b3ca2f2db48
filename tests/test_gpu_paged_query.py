"""GPU parity of dkv_paged_query_attn with the oracle: chunks of different
lengths over whole pages and over a selection's runs.  The pools hold NaN
wherever no token may look: unwritten slots, pruned positions, other pages.

Tolerance: a probability p is used as two bf16 parts, which miss it by at most
2^-9 of the 2^-9 p that the first part leaves, 2^-18 p; n independent such
errors move an output row by less than sqrt(n) 2^-18 of its largest value's
order, and the fp32 sums add some 2^-22 more: sqrt(keys) 2^-17 bounds both."""

import numpy as np
import pytest
import torch

import oracle as o
from _helpers import ATTN_TOL, bits, row_rel_err
from oracle import page_fill as pf

pytestmark = pytest.mark.gpu

DEV = "cuda"
KEEP = 77.0  # what the outputs hold before a call


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEV, dtype=dtype)


def _bf16(rng, shape, scale=1.0):
    return (torch.from_numpy(rng.standard_normal(shape).astype(np.float32)) * scale).to(torch.bfloat16)


class Batch:
    """Sequences that hold held[b] positions and bring new[b] tokens; keep < 1: a selection's runs of the held ones."""

    def __init__(self, rng, held, new, Hkv, G, dim, R, keep=1.0, spare=3, pad=0, fused=True):
        B, self.Hkv, self.G, self.dim, self.R = len(held), Hkv, G, dim, R
        held, new = np.asarray(held), np.asarray(new)
        self.T = int(held.max()) if keep < 1.0 else None
        start = np.full(B, self.T) if keep < 1.0 else held  # position of the first new token
        pps = int((start + new).max()) // R + 1
        S = B * Hkv
        self.pages = S * pps + spare
        self.table = rng.permutation(self.pages)[:S * pps].reshape(S, pps)
        self.k = torch.full((self.pages, R, dim), float("nan"), dtype=torch.bfloat16)
        self.v = self.k.clone()
        if keep < 1.0:
            mask, at = np.zeros((S, self.T), dtype=np.uint8), 0
            while at < self.T:  # runs of positions, some longer than a page
                n = int(rng.integers(1, 3 * R))
                mask[:, at:at + n] = rng.uniform(size=(S, 1)) < keep
                at += n
            mask[np.arange(self.T)[None, :] >= np.repeat(held, Hkv)[:, None]] = 0
            cap = int(new.max()) + 5
            wide = np.concatenate([self.table, self.table[:, :1].repeat(-(-(self.T + cap) // R), 1)], axis=1)
            sel = o.page_select(mask, wide, R, cap)
            lists = sel["entries"]
        else:
            lists = []
            for s in range(S):
                n = int(held[s // Hkv] + new[s // Hkv])
                lists.append([(self.table[s, p], p, 0, min(R, n - p * R)) for p in range(-(-n // R))])
        self.entries = np.full((S, max([1] + [len(x) for x in lists]), 4), -1)
        for s, x in enumerate(lists):
            self.entries[s, :len(x)] = np.array(x).reshape(-1, 4)
            b = s // Hkv
            for page, lp, lo, hi in np.array(x).reshape(-1, 4).tolist():
                hi = max(lo, min(hi, int(start[b] + new[b]) - lp * R))  # what is written so far
                self.k[page, lo:hi] = _bf16(rng, (hi - lo, dim))
                self.v[page, lo:hi] = _bf16(rng, (hi - lo, dim))
        self.n_entries = np.array([len(x) for x in lists])
        self.first_pos, self.new = start.copy(), new
        self.tok_off = np.concatenate([[0], np.cumsum(new)])
        self.tokens, self.max_q = int(new.sum()) + pad, int(new.max()) if B else 0
        x = _bf16(rng, (self.tokens, Hkv * G + (3 if fused else 0), dim))
        self.q_dev = x.to(DEV)[:, (2 if fused else 0):][:, :Hkv * G]
        self.q = x[:, (2 if fused else 0):][:, :Hkv * G]
        self.keys = int((held + new).max())

    def run(self, d, scale=None, hint=None, stream=None, out=None, ws=None):
        scale = 1.0 / np.sqrt(self.dim) if scale is None else scale
        B = len(self.first_pos)
        hint = int(np.maximum(self.n_entries, 0).sum()) * self.R if hint is None else hint
        need = d.dkv_paged_query_workspace_bytes(B, self.Hkv * self.G, self.Hkv, self.dim, self.tokens, self.max_q, hint)
        if ws is None:
            ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device=DEV)
        if out is None:
            out = torch.full((self.tokens, self.Hkv * self.G, self.dim), KEEP, device=DEV)
        if not hasattr(self, "dev"):
            self.dev = (_dev(self.tok_off), _dev(self.first_pos), self.k.to(DEV), self.v.to(DEV), _dev(self.entries),
                        _dev(self.n_entries))
        d.dkv_paged_query_attn(self.q_dev, *self.dev, scale, out, ws, self.Hkv, self.max_q, rows_hint=hint, stream=stream)
        return out

    def want(self, scale=None):
        scale = 1.0 / np.sqrt(self.dim) if scale is None else scale
        kb, vb = bits(self.k.nan_to_num(0.0)), bits(self.v.nan_to_num(0.0))
        n = np.minimum(self.n_entries, self.entries.shape[1])
        w = pf.chunk_attn(bits(self.q), self.tok_off, self.first_pos, kb, vb, self.entries, n, scale, self.Hkv, o.BF16,
                          self.max_q)
        return np.where(np.isnan(w), KEEP, w)

    def check(self, d, tol=None, **kw):
        got = self.run(d, **kw).cpu().numpy()
        want = self.want(kw.get("scale"))
        assert np.isfinite(got).all()
        tol = np.sqrt(max(1, self.keys)) * 2.0 ** -17 if tol is None else tol
        err = row_rel_err(got.reshape(-1, self.dim), want.reshape(-1, self.dim))
        assert err <= tol, (err, tol)
        return got


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("R", [32, 64, 128, 256, 512, 1024])
@pytest.mark.parametrize("G", [1, 3, 4, 7, 8, 16])
def test_random_batches(d, dim, R, G):
    """Whole pages: lengths from nothing on, chunks of one token to many, sequences without any, padded rows."""
    for trial in range(3):
        rng = np.random.default_rng([dim, R, G, trial])
        B = int(rng.integers(1, 6))
        held = rng.choice([0, 1, R - 1, R, R + 1, 300, 700], size=B)
        new = rng.choice([0, 1, 1, 2, 17, 33, 70], size=B)
        new[rng.integers(B)] = rng.choice([1, 5, 40])
        Batch(rng, held, new, int(rng.choice([1, 2, 3])), G, dim, R, pad=int(rng.integers(0, 4)),
              fused=bool(trial % 2)).check(d)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("R", [32, 128, 1024])
@pytest.mark.parametrize("keep", [0.0, 0.03, 0.5])
@pytest.mark.parametrize("new", [[1, 1, 1], [5, 0, 3], [60, 2, 90]])
def test_selected_runs(d, dim, R, keep, new):
    """The entries of a selection: runs that begin and end inside pages, segments with nothing but the new tokens, an
    append region longer than the chunk."""
    rng = np.random.default_rng([dim, R, int(keep * 100), new[0]])
    Batch(rng, [1500, 40, 901], new, 2, 4, dim, R, keep=keep, pad=2).check(d)


@pytest.mark.parametrize("n", [129, 300, 1025])
@pytest.mark.parametrize("R", [32, 64, 256])
def test_prompts_from_their_first_token(d, n, R):
    """Causal from the first position on: token 0 sees itself alone; the last query tiles see far more than the first."""
    rng = np.random.default_rng([n, R])
    Batch(rng, [0, 0, 3], [n, 7, n // 2], 2, 3, 128, R).check(d)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [[1], [4], [9, 1], [20], [30, 2], [50], [61, 33], [65], [200, 1, 3]])
def test_long_contexts(d, dim, new):
    """The keys of a segment are split; unequal lengths, and hints that are wrong."""
    rng = np.random.default_rng([dim, len(new), new[0]])
    held = [20000, 333, 7001][:len(new)]
    x = Batch(rng, held, new, 2, 4, dim, 64)
    want = None
    for hint in (None, 0, 1, 3000, 10 ** 7, 1 << 40):
        got = x.check(d, hint=hint) if want is None else x.run(d, hint=hint).cpu().numpy()
        want = got if want is None else want
        assert row_rel_err(got.reshape(-1, dim), want.reshape(-1, dim)) <= np.sqrt(20200) * 2.0 ** -17, hint


@pytest.mark.parametrize("B,Hkv", [(1, 1), (40, 8), (300, 4), (2048, 1)])
def test_many_single_tokens(d, B, Hkv):
    """A decode step: one token of each of many sequences, some empty."""
    rng = np.random.default_rng(B)
    held = rng.integers(0, 200, size=B)
    Batch(rng, held, np.ones(B, dtype=int), Hkv, 2, 64, 32, pad=1).check(d)


def test_a_decode_step_as_paged_decode(d):
    """Single tokens of equal lengths: what dkv_paged_decode_attn gives, within both kernels' error."""
    rng = np.random.default_rng(5)
    x = Batch(rng, [5000] * 4, [1] * 4, 2, 4, 128, 128, fused=False)
    got = x.check(d)
    out = torch.empty((4, 8, 128), device=DEV)
    ws = torch.empty(d.dkv_decode_workspace_bytes(4, 8, 2, 128), dtype=torch.uint8, device=DEV)
    d.dkv_paged_decode_attn(x.q_dev.contiguous(), x.dev[2], x.dev[3], x.dev[4], x.dev[5], 5001, 0, 1.0 / np.sqrt(128), out,
                            ws, 2)
    assert row_rel_err(got.reshape(-1, 128), out.cpu().numpy().reshape(-1, 128)) <= np.sqrt(5001) * 2.0 ** -17


@pytest.mark.parametrize("new", [[3, 2], [100, 1]])
@pytest.mark.parametrize("scale", [-0.7, 0.0, 3.0])
@pytest.mark.parametrize("held", [150, 6000])
def test_scales(d, scale, new, held):
    """Negative, zero and large: scores of some 200 carry fp32 products' errors into the exponent, so the attention
    tolerance of the other tests holds here."""
    rng = np.random.default_rng([held, new[0]])
    Batch(rng, [held, held // 3], new, 2, 4, 128, 64).check(d, tol=ATTN_TOL, scale=scale)


@pytest.mark.parametrize("new", [[6, 9, 1], [80, 200, 1]])
def test_sequences_that_attend_nothing(d, new):
    """A negative first position, no entries, a count below zero: zeros; a position before every key: zeros."""
    rng = np.random.default_rng(new[0])
    for what in range(4):
        x = Batch(rng, [400, 90, 700], new, 2, 4, 128, 32)
        if what == 0:
            x.first_pos[1] = -1
        elif what == 1:
            x.n_entries[2:4] = [0, -6]
        elif what == 2:  # pages that lie past the chunk
            x.entries[:, :, 1] += 1000
        else:
            x.first_pos[:] = -1
        got = x.check(d)
        if what != 1:
            assert (got[x.tok_off[1]:x.tok_off[2]] == 0).all()


@pytest.mark.parametrize("new", [[6, 9], [80, 140]])
def test_entries_that_name_nothing(d, new):
    """Pages outside the pool, slots outside a page, empty and reversed ranges, page numbers below zero and beyond any
    position, counts above the list's length."""
    rng = np.random.default_rng(new[0] + 1)
    x = Batch(rng, [2000, 1900], new, 2, 4, 64, 32)
    E = x.entries
    for s in range(4):
        E[s, 3, 0], E[s, 5, 0] = -1, x.pages
        E[s, 8, 2:], E[s, 9, 2:], E[s, 10, 2:] = (-1, 20), (5, 33), (20, 20)
        E[s, 11, 2:], E[s, 12, 2:] = (25, 7), (31, 32)
        E[s, 13, 1], E[s, 14, 0] = -13, 2 ** 31 - 1
        E[s, 7, 2:] = (3, 29)
    x.n_entries[1], x.n_entries[2] = E.shape[1] + 100, 11
    E[0, 15:, 1] = 2 ** 31 - 1  # position past the largest: hidden, and so is what follows
    x.check(d)


def test_offsets_that_do_not_fit(d):
    """Token offsets below zero, past the rows, decreasing; a chunk longer than max_q: the rows that belong to a
    sequence are right, all others stay."""
    rng = np.random.default_rng(9)
    x = Batch(rng, [300, 200, 100, 50], [20, 30, 10, 5], 2, 4, 128, 32)
    x.max_q = 25
    x.check(d)
    y = Batch(rng, [300, 200], [20, 30], 2, 4, 128, 32)
    full = y.check(d)
    del y.dev
    y.tok_off = np.array([20, 90])  # runs past the rows
    y.first_pos, y.entries, y.n_entries = y.first_pos[1:], y.entries[2:], y.n_entries[2:]
    got = y.run(d).cpu().numpy()
    np.testing.assert_array_equal(got[:20], KEEP)
    assert row_rel_err(got[20:].reshape(-1, 128), full[20:].reshape(-1, 128)) <= np.sqrt(330) * 2.0 ** -17
    for off in ([30, 20], [-5, 10], [60, 70], [50, 50], [2 ** 31 - 1, -2 ** 31]):
        del y.dev
        y.tok_off = np.array(off)
        np.testing.assert_array_equal(y.run(d).cpu().numpy(), KEEP)


def test_positions_up_to_the_largest(d):
    """Chunks at the end of the 31-bit positions: pages there are attended, and nothing wraps."""
    rng = np.random.default_rng(10)
    for n in (3, 100):
        x = Batch(rng, [300], [n], 2, 4, 128, 32)
        shift = (2 ** 31 - 1) // 32 - 20
        x.entries[:, :, 1] += shift
        x.first_pos += shift * 32
        x.check(d)


def test_pools_past_4_gib(d):
    """Pages whose byte offsets pass 32 bits give what the same rows near the start give, bit for bit."""
    rng = np.random.default_rng(12)
    for new in ([3, 1], [150, 1]):
        x = Batch(rng, [600, 90], new, 2, 4, 128, 1024)
        want = x.run(d)
        far, pages = 36000, 36000 + x.pages
        k = torch.empty((pages, 1024, 128), dtype=torch.bfloat16, device=DEV)
        v = torch.empty_like(k)
        k[far:], v[far:] = x.dev[2], x.dev[3]
        x.dev = (*x.dev[:2], k, v, x.dev[4] + _dev([far, 0, 0, 0]), x.dev[5])
        assert torch.equal(x.run(d), want)
        del k, v, x
        torch.cuda.empty_cache()


@pytest.mark.parametrize("new", [[1] * 6, [70, 1, 1, 9, 1, 1]])
def test_replays_of_two_graphs(d, new):
    """Two captured calls with workspaces of their own, replayed by turns with eager calls and new inputs between."""
    rng = np.random.default_rng(14)
    held = [9000, 20, 300, 64, 0, 1200]
    x, y = (Batch(rng, held, new, 2, 4, 128, 64) for _ in range(2))
    want = [z.run(d).clone() for z in (x, y)]
    graphs = []
    for z in (x, y):
        need = max(16, d.dkv_paged_query_workspace_bytes(6, 8, 2, 128, z.tokens, z.max_q, int(z.n_entries.sum()) * 64))
        ws = torch.empty(need, dtype=torch.uint8, device=DEV)
        out = torch.full((z.tokens, 8, 128), KEEP, device=DEV)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            z.run(d, out=out, ws=ws)
        graphs.append((g, out, ws))
    for i in range(4):
        for (g, out, _), w, z in zip(graphs, want, (x, y)):
            out.fill_(KEEP)
            g.replay()
            assert torch.equal(z.run(d), w)
            assert torch.equal(out, w), i


def test_another_stream(d):
    """The call runs on the stream that it is given, and on the current one."""
    rng = np.random.default_rng(15)
    x = Batch(rng, [5000, 100], [40, 1], 2, 4, 128, 64)
    want = x.run(d)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = x.run(d, stream=s)
    with torch.cuda.stream(s):
        again = x.run(d)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(again, want)


def test_the_same_call_gives_the_same_bits(d):
    rng = np.random.default_rng(16)
    x = Batch(rng, [9000, 100, 4000], [300, 1, 20], 2, 4, 128, 64)
    want = x.run(d)
    for _ in range(5):
        assert torch.equal(x.run(d), want)


@pytest.mark.parametrize("R", [32, 128])
def test_a_server_from_prompts_to_release(d, R):
    """The calls together, on the GPU alone: prompts in chunks (extend, append, attend), then single tokens; a
    selection of the context, its unused pages released, and a question to what is left; the pages go to a new
    request.  Checked against the oracle's dense attention from the positions."""
    rng = np.random.default_rng(R)
    B, Hkv, G, dim = 3, 2, 4, 128
    Hq, S, scale = Hkv * G, B * Hkv, 1.0 / np.sqrt(128)
    chunks = [[90, 75, 1], [110, 1, 100], [1, 1, 31], [1, 1, 1]]
    total = np.array(chunks).sum(axis=0)
    pps, pages = int(total.max()) // R + 4, S * (int(total.max()) // R + 4)
    i32 = lambda *s: torch.full(s, -1, dtype=torch.int32, device=DEV)  # noqa: E731
    stack, n_free = _dev(rng.permutation(pages)), _dev([pages])
    table, entries, counts = i32(S, pps), i32(S, pps, 4), torch.zeros(S, dtype=torch.int32, device=DEV)
    length, tok_off, first_pos = torch.zeros(B, dtype=torch.int32, device=DEV), i32(B + 1), i32(B)
    k_pages = torch.full((pages, R, dim), float("nan"), dtype=torch.bfloat16, device=DEV)
    v_pages = torch.full_like(k_pages, float("nan"))
    ews = torch.empty(d.dkv_page_extend_workspace_bytes(B), dtype=torch.uint8, device=DEV)
    hist = [(np.zeros((Hkv, 0, dim)), np.zeros((Hkv, 0, dim))) for _ in range(B)]

    def attend(x, tokens, most, ent, cnt):
        need = d.dkv_paged_query_workspace_bytes(B, Hq, Hkv, dim, tokens, most, 0)
        ws = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
        out = torch.empty((tokens, Hq, dim), device=DEV)
        d.dkv_paged_query_attn(x[:, :Hq], tok_off, first_pos, k_pages, v_pages, ent, cnt, scale, out, ws, Hkv, most)
        return out.cpu().numpy()

    def expect(x, new, kept=None):
        rows, at = [], 0
        for b, n in enumerate(new):
            xb = x[at:at + n].double().numpy()
            for j in range(2):
                add = xb[:, Hq + j * Hkv:Hq + (j + 1) * Hkv].transpose(1, 0, 2)
                old = hist[b][j]
                hist[b] = (np.concatenate([old, add], axis=1), hist[b][1]) if j == 0 else (
                    hist[b][0], np.concatenate([old, add], axis=1))
            for t in range(n):
                ctx = hist[b][0].shape[1] - n
                see = ctx + t + 1
                row = np.zeros((Hq, dim))
                for h in range(Hq):
                    g = h // G
                    m = np.ones(see, dtype=bool)
                    if kept is not None:
                        m[:ctx] = kept[b * Hkv + g][:ctx] != 0
                    s = scale * hist[b][0][g, :see][m] @ xb[t, h]
                    p = np.exp(s - s.max())
                    row[h] = p @ hist[b][1][g, :see][m] / p.sum()
                rows.append(row)
            at += n
        return np.array(rows)

    for new in chunks:
        tokens, most = sum(new), max(new)
        x = _bf16(rng, (tokens, Hq + 2 * Hkv, dim))
        xd = x.to(DEV)
        slots = torch.full((tokens, Hkv), -5, dtype=torch.int64, device=DEV)
        d.dkv_page_extend(_dev(new), length, stack, n_free, table, R, Hkv, tok_off, first_pos, slots, ews, entries=entries,
                          n_entries=counts)
        d.dkv_paged_append(xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], slots, k_pages, v_pages)
        got = attend(xd, tokens, most, entries, counts)
        want = expect(x, new)
        assert row_rel_err(got.reshape(-1, dim), want.reshape(-1, dim)) <= np.sqrt(300) * 2.0 ** -17
    assert length.cpu().tolist() == total.tolist()

    # room for a question's tokens, a selection of the context, its pages back
    T, n_q = int(total.max()), 6
    grow = _dev(T + n_q - total)
    slots = torch.empty((int((T + n_q - total).sum()), Hkv), dtype=torch.int64, device=DEV)
    d.dkv_page_extend(grow, length, stack, n_free, table, R, Hkv, tok_off, first_pos, slots, ews)
    keep = (rng.uniform(size=(S, T)) < 0.3).astype(np.uint8)
    keep[:, 40:40 + 2 * R] = 0
    keep[np.arange(T)[None, :] >= np.repeat(total, Hkv)[:, None]] = 0
    flat = torch.zeros(S * T + 16, dtype=torch.uint8, device=DEV)
    mask = flat[:S * T].view(S, T)
    mask.copy_(_dev(keep, torch.uint8))
    max_e = 40 + T // 2
    ent, cnt, seg_len = i32(S, max_e, 4), i32(S), i32(S)
    used = torch.empty((S, pps), dtype=torch.uint8, device=DEV)
    sws = torch.empty(max(16, d.dkv_page_select_workspace_bytes(S, T)), dtype=torch.uint8, device=DEV)
    d.dkv_page_select(mask, table, R, n_q, ent, cnt, seg_len, sws, page_used=used)
    before, unused = int(n_free), int(((used == 0) & (table >= 0)).sum())
    rws = torch.empty(d.dkv_page_release_workspace_bytes(S, pps), dtype=torch.uint8, device=DEV)
    d.dkv_page_release(table, stack, n_free, rws, keep=used)
    assert int(n_free) == before + unused
    freed = stack[before:int(n_free)].long()
    k_pages[freed], v_pages[freed] = float("nan"), float("nan")
    x = _bf16(rng, (B * n_q, Hq + 2 * Hkv, dim))
    xd = x.to(DEV)
    pos = T + torch.arange(n_q, device=DEV)
    page = table.long()[:, pos // R].view(B, Hkv, n_q)
    slots = (page * R + pos % R).permute(0, 2, 1).reshape(B * n_q, Hkv).contiguous()
    d.dkv_paged_append(xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], slots, k_pages, v_pages)
    tok_off.copy_(_dev(np.arange(B + 1) * n_q))
    first_pos.copy_(_dev([T] * B))
    got = attend(xd, B * n_q, n_q, ent, cnt)
    want = expect(x, [n_q] * B, keep)
    assert row_rel_err(got.reshape(-1, dim), want.reshape(-1, dim)) <= np.sqrt(300) * 2.0 ** -17
    want_free = int(n_free)
    new_len = torch.zeros(1, dtype=torch.int32, device=DEV)
    t2, off2, pos2 = i32(Hkv, pps), i32(2), i32(1)
    slots = torch.empty((R + 1, Hkv), dtype=torch.int64, device=DEV)
    d.dkv_page_extend(_dev([R + 1]), new_len, stack, n_free, t2, R, Hkv, off2, pos2, slots, ews)
    assert int(n_free) == want_free - 2 * Hkv and int(pos2) == 0 and (slots >= 0).all()


@pytest.mark.parametrize("dim,G,Hkv,B,new", [(64, 4, 2, 40, 300), (128, 4, 2, 40, 300), (128, 7, 4, 13, 260),
                                             (64, 8, 8, 256, 66)])
@pytest.mark.parametrize("held", [0, 90])
def test_many_prompts(d, dim, G, Hkv, B, new, held):
    """More query tiles than compute units, none with more than a workgroup's share of the keys; more of them than a
    workgroup sorts."""
    rng = np.random.default_rng([dim, B, new, held])
    new = rng.integers(new - new // 10, new + 1, size=B)
    Batch(rng, rng.integers(0, held + 1, size=B), new, Hkv, G, dim, 64, pad=1).check(d)


@pytest.mark.parametrize("dim,G,B,new,held", [(64, 16, 40, 320, 700), (128, 7, 64, 290, 500)])
def test_many_long_query_tiles(d, dim, G, B, new, held):
    """Enough tiles of enough keys that workgroups take them whole, round by round."""
    rng = np.random.default_rng([dim, B, held])
    new = rng.integers(new - 60, new + 1, size=B)
    Batch(rng, rng.integers(held - 100, held + 1, size=B), new, 1, G, dim, 128).check(d)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("held", [32768 - 70, 32768 - 16, 33000])
def test_contexts_around_the_third_part(d, dim, held):
    """Query tiles that see 32,768 rows and more, in which a probability has two parts instead of three."""
    rng = np.random.default_rng([dim, held])
    Batch(rng, [held, 40], [17, 20], 1, 16, dim, 1024).check(d)


@pytest.mark.parametrize("dim,R", [(64, 32), (128, 32), (128, 64)])
@pytest.mark.parametrize("new", [17, 20, 33])
def test_one_workgroup_walks_a_long_context(d, dim, R, new):
    """A hint of one row: no split, and more runs than their table holds at a time; last tiles of one row group to
    all."""
    rng = np.random.default_rng([dim, R, new])
    x = Batch(rng, [80001 * R // 32, 5], [new, 18], 1, 16, dim, R)
    got = x.check(d, hint=1)
    split = x.run(d).cpu().numpy()
    assert row_rel_err(split.reshape(-1, dim), got.reshape(-1, dim)) <= np.sqrt(x.keys) * 2.0 ** -17


@pytest.mark.parametrize("new", [[70] + [66] * 9, [1] * 20, [9] + [3] * 30])
@pytest.mark.parametrize("long", [2100, 25000])
def test_one_long_sequence_among_short_ones(d, new, long):
    rng = np.random.default_rng([len(new), long])
    held = rng.integers(0, 40, size=len(new))
    held[len(new) // 2] = long
    Batch(rng, held, new, 2, 4, 128, 64).check(d)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("R", [32, 256])
@pytest.mark.parametrize("B,n,held", [(1, 64, 9000), (3, 30, 2500), (12, 31, 3000), (30, 17, 600), (4, 40, 5000)])
def test_blocks_between_the_kernels(d, dim, R, B, n, held):
    """65 to 256 query rows of few long and of many short segments."""
    rng = np.random.default_rng([dim, R, B])
    new = rng.integers(1, n + 1, size=B)
    new[0] = n
    Batch(rng, rng.integers(held // 2, held + 1, size=B), new, 2, 4, dim, R).check(d)


@pytest.mark.parametrize("new,held", [([1] * 5, 3000), ([80, 3], 9000), ([30, 10], 4000), ([300] * 40, 0), ([200], 0)])
@pytest.mark.parametrize("hint", [None, 0, 1, 50000])
def test_writes_stay_in_the_workspace_and_the_output(d, new, held, hint):
    rng = np.random.default_rng([len(new), held])
    x = Batch(rng, [held] * len(new), new, 2, 4, 64, 64)
    h = int(x.n_entries.sum()) * 64 if hint is None else hint
    need = d.dkv_paged_query_workspace_bytes(len(new), 8, 2, 64, x.tokens, x.max_q, h)
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    buf = torch.full((x.tokens + 8, 8, 64), KEEP, device=DEV)
    x.run(d, hint=hint, ws=ws[:max(need, 16)], out=buf[4:4 + x.tokens])
    assert (ws[max(need, 16):] == 0xA5).all()
    assert (buf[:4] == KEEP).all() and (buf[-4:] == KEEP).all()
    assert torch.equal(buf[4:-4], x.run(d, hint=hint))


def test_two_calls_at_once(d):
    """Two streams, workspaces of their own: each gives what it gives alone."""
    rng = np.random.default_rng(21)
    x = Batch(rng, [9000, 20, 300], [150, 1, 9], 2, 4, 128, 64)
    y = Batch(rng, [7000, 5000], [40, 40], 2, 4, 128, 32)
    want = [z.run(d) for z in (x, y)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(6):
        for z, s in zip((x, y), streams):
            with torch.cuda.stream(s):
                got.append(z.run(d))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert torch.equal(g, want[i % 2]), i


def test_a_sequence_listed_twice(d):
    """Two sequences that read the same pages, as requests with a common prefix do, at different positions."""
    rng = np.random.default_rng(22)
    x = Batch(rng, [3000, 3000], [50, 50], 2, 4, 128, 64)
    x.entries[2:] = x.entries[:2]
    x.first_pos[1] = 1500
    x.check(d)


@pytest.mark.parametrize("n", [1, 40, 300])
def test_a_padded_batch_replayed_with_other_lengths(d, n):
    """One captured call whose offsets, positions and lists are rewritten between replays: sequences come and go, rows
    behind the last one stay."""
    rng = np.random.default_rng([23, n])
    shapes = [([900, 40, 7], [n, 1, 1]), ([0, 0, 0], [0, 0, n]), ([3000, 1, 2000], [1, n, 0]), ([5, 5, 5], [0, 0, 0])]
    batches = [Batch(rng, h, w, 2, 4, 128, 64, pad=n + 2 - sum(w), fused=False) for h, w in shapes]
    pages, wide = max(b.pages for b in batches), max(b.entries.shape[1] for b in batches)
    hold = [torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV),
            torch.zeros((pages, 64, 128), dtype=torch.bfloat16, device=DEV),
            torch.zeros((pages, 64, 128), dtype=torch.bfloat16, device=DEV),
            torch.zeros((6, wide, 4), dtype=torch.int32, device=DEV), torch.zeros(6, dtype=torch.int32, device=DEV)]
    q = torch.zeros((n + 2, 8, 128), dtype=torch.bfloat16, device=DEV)
    out = torch.zeros((n + 2, 8, 128), device=DEV)
    ws = torch.empty(d.dkv_paged_query_workspace_bytes(3, 8, 2, 128, n + 2, n, 0), dtype=torch.uint8, device=DEV)
    call = lambda: d.dkv_paged_query_attn(q, *hold, 1.0 / np.sqrt(128), out, ws, 2, n)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in (0, 1, 2, 3, 2, 0):
        b = batches[i]
        q.copy_(b.q_dev)
        hold[0].copy_(_dev(b.tok_off))
        hold[1].copy_(_dev(b.first_pos))
        hold[2][:b.pages].copy_(b.k)
        hold[3][:b.pages].copy_(b.v)
        hold[4][:, :b.entries.shape[1]].copy_(_dev(b.entries))
        hold[5].copy_(_dev(b.n_entries))
        out.fill_(KEEP)
        g.replay()
        got = out.cpu().numpy()
        b.max_q = n
        err = row_rel_err(got.reshape(-1, 128), b.want().reshape(-1, 128))
        assert np.isfinite(got).all() and err <= np.sqrt(3100) * 2.0 ** -17, (i, err)


@pytest.mark.parametrize("dim,R", [(64, 256), (128, 1024), (128, 32)])
@pytest.mark.parametrize("keep,new,held", [(0.3, [20, 17], 9000), (0.02, [150, 3], 9000), (0.5, [18], 70000),
                                           (0.9, [40] * 12, 600)])
def test_query_tiles_over_a_selection(d, dim, R, keep, new, held):
    """Runs without slots between the kept ones, in ranges that fit a table of runs and in longer ones."""
    rng = np.random.default_rng([dim, R, held, len(new)])
    x = Batch(rng, [held] * len(new), new, 1, 16, dim, R, keep=keep, pad=1)
    got = x.check(d)
    whole = x.run(d, hint=1).cpu().numpy()
    assert row_rel_err(whole.reshape(-1, dim), got.reshape(-1, dim)) <= np.sqrt(x.keys) * 2.0 ** -17
