"""GPU parity of dkv_paged_tree_attn with the oracle: trees, chains and general
masks of new tokens over whole pages and over a selection's runs, in bf16 and
quantised.  The pools hold NaN (and its exponent bytes) wherever no token may
look: unwritten slots, pruned positions, other pages.

Tolerance, of a row against its weighted sum of |v|: the products q k and the
probabilities' three parts are exact to 24 bits, so what is left are fp32 sums: a
score's, d roundings of 2^-24 of at most a = scale sum |q k| that add up like a
random walk, with a factor of four; the exponential and the parts, 2^-20; and the
sums over the keys, a random walk of 2^-24 each, with the same factor."""

import numpy as np
import pytest
import torch

from oracle import tree_cache as tc

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


def random_mask(rng, new, tokens, words, kind):
    """uint64 [tokens][words]: "tree", "any" (each bit by chance, tokens after one's own among them) or "none" set."""
    if kind == "tree":
        off = np.concatenate([[0], np.cumsum(new)])
        parent = np.concatenate([rng.integers(np.maximum(-1, np.arange(s) - 5), np.maximum(np.arange(s), 0)) if s else
                                 np.zeros(0, np.int64) for s in new] + [np.zeros(tokens - off[-1], np.int64)])
        return tc.tree_plan(off, np.zeros(len(new)), max(1, max(new)), tokens, parent, words)[1]
    if kind == "none":
        return np.zeros((tokens, words), dtype=np.uint64)
    bits = (rng.uniform(size=(tokens, words * 64)) < rng.choice([0.05, 0.5, 0.95], size=(tokens, 1))).astype(np.uint8)
    return np.packbits(bits, axis=1, bitorder="little").view(np.uint64).reshape(tokens, words)


class Batch:
    """Sequences that hold held[b] positions and bring new[b] tokens; keep < 1: a selection's runs of the held ones."""

    def __init__(self, rng, fmt, held, new, Hkv, G, dim, R, keep=1.0, mask="tree", spare=3, pad=0, extra_words=0, kscale=1.0,
                 vsizes=(1e-3, 1.0, 30.0)):
        B, self.Hkv, self.G, self.dim, self.R, self.fmt = len(held), Hkv, G, dim, R, fmt
        held, new = np.asarray(held), np.asarray(new)
        start = np.full(B, int(held.max())) if keep < 1.0 else held
        pps = int((start + new).max()) // R + 1
        S = B * Hkv
        self.pages = S * pps + spare
        table = rng.permutation(self.pages)[:S * pps].reshape(S, pps)
        f8 = fmt == "f8"
        self.k = np.full((self.pages, R, dim), np.nan)       # values
        self.v = self.k.copy()
        codes = [np.full((self.pages, R, dim), 0x7F, dtype=np.uint8) for _ in range(2)]
        exps = np.full((self.pages, R, 2), 0xFF, dtype=np.uint8)
        lists = []
        for s in range(S):
            T, n = int(start[s // Hkv]), int(new[s // Hkv])
            kept = np.ones(T, dtype=bool)
            if keep < 1.0:
                at = 0
                while at < T:
                    w = int(rng.integers(1, 3 * R))
                    kept[at:at + w] = rng.uniform() < keep
                    at += w
            kept = np.concatenate([kept, np.ones(n, dtype=bool)])
            runs = []
            for p in range(-(-(T + n) // R)):
                edge = np.flatnonzero(np.diff(np.concatenate([[0], kept[p * R:(p + 1) * R].astype(np.int8), [0]])))
                runs += [(table[s, p], p, lo, hi) for lo, hi in edge.reshape(-1, 2).tolist()]
            lists.append(runs)
            for page, _, lo, hi in runs:
                for i, pool in enumerate((self.k, self.v)):
                    x = rng.standard_normal((hi - lo, dim)) * (kscale if i == 0 else rng.choice(vsizes, size=(hi - lo, 1)))
                    if f8:
                        c, e = tc.quantise(x)
                        codes[i][page, lo:hi], exps[page, lo:hi, i] = c, e
                        pool[page, lo:hi] = tc.row_values(c, e)
                    else:
                        pool[page, lo:hi] = torch.from_numpy(x).bfloat16().double().numpy()
        most = max([1] + [len(x) for x in lists])
        self.entries = np.full((S, most, 4), -1)
        for s, x in enumerate(lists):
            self.entries[s, :len(x)] = np.array(x).reshape(-1, 4)
        self.n_entries = np.array([len(x) for x in lists])
        self.first_pos, self.new = start.copy(), new
        self.tok_off = np.concatenate([[0], np.cumsum(new)])
        self.tokens, self.max_q = int(new.sum()) + pad, int(new.max())
        words = -(-max(1, self.max_q) // 64) + extra_words
        self.mask = None if mask is None else random_mask(rng, new, self.tokens, words, mask)
        x = _bf16(rng, (self.tokens, Hkv * G + 3, dim))
        self.q, self.q_dev = x[:, 2:2 + Hkv * G], x.to(DEV)[:, 2:2 + Hkv * G]
        if f8:
            pools = [torch.from_numpy(c).to(DEV).view(torch.float8_e4m3fn) for c in codes]
            self.scales = torch.from_numpy(exps).to(DEV)
        else:
            pools, self.scales = [torch.from_numpy(p).bfloat16().to(DEV) for p in (self.k, self.v)], None
        self.pools = pools
        self.keys = int((held + new).max())

    def run(self, d, scale=None, hint=None, stream=None, out=None, ws=None, mask="own"):
        scale = 1.0 / np.sqrt(self.dim) if scale is None else scale
        B = len(self.first_pos)
        hint = int(np.maximum(self.n_entries, 0).sum()) * self.R if hint is None else hint
        fmt = d.DKV_CACHE_F8 if self.fmt == "f8" else d.DKV_CACHE_BF16
        need = d.dkv_paged_tree_workspace_bytes(fmt, B, self.Hkv * self.G, self.Hkv, self.dim, self.tokens, self.max_q, hint)
        if ws is None:
            ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device=DEV)
        if out is None:
            out = torch.full((self.tokens, self.Hkv * self.G, self.dim), KEEP, device=DEV)
        if not hasattr(self, "dev"):
            self.dev = (_dev(self.tok_off), _dev(self.first_pos), *self.pools, _dev(self.entries), _dev(self.n_entries))
            self.mask_dev = None if self.mask is None else torch.from_numpy(self.mask.view(np.int64)).to(DEV)
        d.dkv_paged_tree_attn(self.q_dev, *self.dev, scale, out, ws, self.Hkv, self.max_q,
                              mask=self.mask_dev if mask == "own" else mask, scales=self.scales, rows_hint=hint, stream=stream)
        return out

    def want(self, scale=None):
        scale = 1.0 / np.sqrt(self.dim) if scale is None else scale
        k, v = np.nan_to_num(self.k), np.nan_to_num(self.v)
        q = self.q.double().numpy()
        n = np.minimum(self.n_entries, self.entries.shape[1])
        args = (self.tok_off, self.first_pos)
        rest = (self.R, self.entries, n, scale, self.Hkv, self.max_q, self.mask)
        out = tc.tree_attn(q, *args, k, v, *rest)
        size = np.nan_to_num(tc.tree_attn(q, *args, k, np.abs(v), *rest)).max(axis=2)
        # the largest scale sum |q k| of a row (over all keys of the pools)
        big = abs(scale) * np.abs(q).max(axis=2) * np.abs(k).sum(axis=2).max()
        return np.where(np.isnan(out), KEEP, out), size, big

    def check(self, d, **kw):
        got = self.run(d, **kw).double().cpu().numpy()
        want, size, big = self.want(kw.get("scale"))
        assert np.isfinite(got).all()
        tol = (4 * np.sqrt(self.dim) * big + 16 + 4 * np.sqrt(self.keys)) * 2.0 ** -24 * size
        err = np.abs(got - want).max(axis=2)
        bad = err > tol
        assert not bad.any(), (np.argwhere(bad)[:5], err[bad][:5], tol[bad][:5])
        return got


FMTS = ["f8", "bf16"]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [[1], [2], [5], [9], [17], [40], [70]])
def test_one_sequence(d, fmt, dim, new):
    """Every kernel's share of rows, one short sequence, no mask and a tree."""
    for G in (1, 4, 7):
        for mask in (None, "tree"):
            rng = np.random.default_rng([dim, new[0], G])
            Batch(rng, fmt, [45], new, 1, G, dim, 32, mask=mask).check(d)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("R", [32, 64, 128, 1024])
@pytest.mark.parametrize("G", [1, 3, 4, 8, 16])
def test_random_batches(d, fmt, dim, R, G):
    """Whole pages: lengths from nothing on, trees of one token to many, sequences without any, padded rows."""
    for trial, mask in enumerate(("tree", "any", None)):
        rng = np.random.default_rng([dim, R, G, trial])
        B = int(rng.integers(1, 6))
        held = rng.choice([0, 1, R - 1, R, R + 1, 300, 700], size=B)
        new = rng.choice([0, 1, 2, 17, 33, 70], size=B)
        new[rng.integers(B)] = rng.choice([1, 5, 40])
        Batch(rng, fmt, held, new, int(rng.choice([1, 2, 3])), G, dim, R, mask=mask, pad=int(rng.integers(0, 4)),
              extra_words=trial % 2).check(d)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("R", [32, 128, 1024])
@pytest.mark.parametrize("new", [[1, 1, 1], [5, 0, 3], [60, 2, 90]])
def test_selected_runs(d, fmt, dim, R, new):
    """The entries of a selection: runs that begin and end inside pages, segments with nothing but the new tokens."""
    for keep in (0.0, 0.03, 0.5):
        for mask in ("tree", None):
            rng = np.random.default_rng([dim, R, sum(new), int(100 * keep)])
            Batch(rng, fmt, [900, 500, 1], new, 2, 4, dim, R, keep=keep, mask=mask).check(d)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 6, 16, 30, 64, 150])
def test_long_split(d, fmt, dim, new):
    """Long segments: keys split over workgroups and joined; an exact, a wrong, a huge and no hint."""
    rng = np.random.default_rng([dim, new])
    b = Batch(rng, fmt, [20000, 3000], [new, max(1, new // 2)], 2, 4, dim, 128, mask="tree")
    want, size, big = b.want()
    tol = (4 * np.sqrt(dim) * big + 16 + 4 * np.sqrt(b.keys)) * 2.0 ** -24 * size
    exact = int(b.n_entries.sum()) * 128
    for hint in (exact, exact // 7, 1 << 45, 0, 1):
        got = b.run(d, hint=hint).double().cpu().numpy()
        assert (np.abs(got - want).max(axis=2) <= tol).all(), hint


@pytest.mark.parametrize("fmt", FMTS)
def test_rows_that_see_nothing(d, fmt):
    """Masks that leave nothing, over no context and a context; sequences marked as attending nothing."""
    for dim, G, n in ((64, 4, 5), (128, 8, 20), (128, 4, 100)):
        rng = np.random.default_rng([dim, n])
        b = Batch(rng, fmt, [0, 40, 0, 33], [n, n, 1, 2], 2, G, dim, 32, mask="none")
        b.first_pos[3] = -1
        got = b.check(d)
        assert (got[:n] == 0).all() and (got[2 * n:] == 0).all() and (got[n:2 * n] != 0).any()
        b = Batch(rng, fmt, [0, 40], [n, n], 2, G, dim, 32, mask="any")
        b.mask[::2] = 0
        b.check(d)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("new", [3, 30, 90, 300])
def test_chain_mask_equals_no_mask(d, fmt, new):
    rng = np.random.default_rng(new)
    b = Batch(rng, fmt, [500, 1000, 3], [new, 1, max(1, new // 3)], 2, 4, 128, 64, mask="none")
    b.mask = tc.tree_plan(b.tok_off, b.first_pos, b.max_q, b.tokens, None, b.mask.shape[1])[1]
    got = b.run(d)
    again = b.run(d, mask=None)
    # the keys may be cut into other slices, as a masked tile of rows sees the whole chunk
    assert (got - again).abs().max() <= 2.0 ** -18 * got.abs().max()
    b.check(d)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 12, 50, 200])
def test_bf16_chains_are_the_chunk_call(d, dim, new):
    """Without a mask, over bf16 pools, the call is dkv_paged_query_attn's, bit for bit."""
    rng = np.random.default_rng([dim, new])
    b = Batch(rng, "bf16", [3000, 20], [new, 1], 2, 4, dim, 128, mask=None)
    got = b.run(d)
    hint = int(b.n_entries.sum()) * 128
    out = torch.full_like(got, KEEP)
    ws = torch.zeros(1 << 26, dtype=torch.uint8, device=DEV)
    d.dkv_paged_query_attn(b.q_dev, *b.dev, 1.0 / np.sqrt(dim), out, ws, 2, b.max_q, rows_hint=hint)
    assert torch.equal(got, out)


@pytest.mark.parametrize("fmt", FMTS)
def test_scales_and_large_logits(d, fmt):
    for scale, kscale in ((-0.2, 1.0), (0.0, 1.0), (1.0, 6.0), (1e-30, 1.0)):
        for n in (2, 20, 90):
            rng = np.random.default_rng(n)
            Batch(rng, fmt, [300], [n], 1, 4, 128, 64, kscale=kscale).check(d, scale=scale)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 10, 40, 200])
def test_rows_of_v_far_apart(d, fmt, dim, n):
    """Rows of zeros and of 2^-40 beside rows of 1 and of 2^20, at probabilities that differ as much: a key's share of the
    sum must not depend on the size of its V (the share of one of 2^-60 beside one of 2^24 counts down to 2^-49, beyond
    the tolerance); one or two large rows among zeros."""
    for vsizes in ((0.0, 2.0 ** -40, 1.0, 2.0 ** 20), (0.0,) * 60 + (100.0,), (0.0,)):
        rng = np.random.default_rng([dim, n])
        b = Batch(rng, fmt, [900, 3], [n, 1], 2, 4, dim, 64, kscale=1.5, vsizes=vsizes)
        got = b.check(d, scale=0.7)
        assert vsizes != (0.0,) or (got == 0).all()


@pytest.mark.parametrize("n", [1, 10, 40, 200])
def test_scores_beyond_the_range_stay_finite(d, n):
    """Quantised, scores of 2^25 to 2^100: which keys win is lost to rounding, but nothing overflows."""
    for scale in (1e6, -1e12, 1e30):
        b = Batch(np.random.default_rng(n), "f8", [700], [n], 1, 4, 128, 64)
        assert torch.isfinite(b.run(d, scale=scale)).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_bad_entries_and_offsets(d, fmt):
    """Entries outside the pool or a page attend nothing; offsets that do not fit give fewer tokens; max_q cuts."""
    for n in (3, 30, 100):
        rng = np.random.default_rng(n)
        b = Batch(rng, fmt, [200, 130], [n, n], 2, 4, 128, 32)
        b.entries[0, 1] = (b.pages, 1, 0, 32)
        b.entries[1, 2] = (-1, 2, 0, 32)
        b.entries[2, 0] = (b.entries[2, 0][0], 0, 0, 33)
        b.entries[3, 1] = (b.entries[3, 1][0], 1, -1, 32)
        b.check(d)
        b.max_q = n - 1
        b.check(d)
        b.tok_off = np.array([0, n, 10 ** 9])  # taken within the rows
        b.max_q = n
        b.check(d)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n", [1, 20, 64])
def test_positions_at_the_end(d, fmt, n):
    """Logical pages whose positions end at 2^31 - 1."""
    rng = np.random.default_rng(n)
    b = Batch(rng, fmt, [90], [n], 1, 4, 64, 32, mask="tree")
    shift = (2 ** 31 - 1 - 90 - n) // 32
    b.entries[..., 1] += shift
    b.first_pos = b.first_pos + shift * 32
    b.check(d)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n, held", [(1, 5000), (24, 9000), (100, 2000)])
def test_repeats_streams_and_graphs(d, fmt, n, held):
    """The same bits call after call, on another stream, and from a graph replayed with eager work in between."""
    rng = np.random.default_rng(n)
    b = Batch(rng, fmt, [held, 700], [n, 1], 2, 4, 128, 128)
    first = b.run(d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = b.run(d, stream=s)
    s.synchronize()
    assert torch.equal(first, other) and torch.equal(first, b.run(d))
    ws = torch.full((1 << 26,), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full_like(first, KEEP)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        b.run(d, out=out, ws=ws)
    for i in range(4):
        out.fill_(KEEP)
        ws.fill_(i)
        g.replay()
        assert torch.equal(out, first)
        assert torch.equal(b.run(d), first)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n, held", [(1, 4000), (9, 4000), (40, 4000), (300, 1000)])
def test_precision(d, fmt, n, held):
    """Three parts of a probability: an output is within 10^-6 of its norm (two would err by 2.1e-6 and more)."""
    rng = np.random.default_rng(n)
    b = Batch(rng, fmt, [held], [n], 1, 4, 128, 128)
    got = b.run(d).double().cpu().numpy()
    want, _, _ = b.want()
    assert np.linalg.norm(got - want) <= 1e-6 * np.linalg.norm(want)


@pytest.mark.parametrize("fmt", FMTS)
def test_pool_beyond_2_31(d, fmt):
    """Pages whose offsets pass 2^31 bytes and elements."""
    dim, R, Hkv, G, n = 128, 1024, 1, 4, 9
    rng = np.random.default_rng(5)
    small = Batch(rng, fmt, [3000], [n], Hkv, G, dim, R)
    want = small.run(d)
    pages = (1 << 32) // (R * dim * (1 if fmt == "f8" else 2)) + 40
    big = []
    for x in small.pools + ([small.scales] if fmt == "f8" else []):
        y = torch.zeros((pages, *x.shape[1:]), dtype=x.dtype, device=DEV)
        y.view(torch.uint8)[pages - small.pages:] = x.view(torch.uint8)
        big.append(y)
    small.entries[..., 0] += pages - small.pages
    small.pools, small.scales = big[:2], big[2] if fmt == "f8" else None
    del small.dev
    assert torch.equal(small.run(d), want)
