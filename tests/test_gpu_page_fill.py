"""GPU parity of dkv_page_extend, dkv_page_release and dkv_paged_append with
the oracle, bit for bit: every output whole, what is not written included."""

import numpy as np
import pytest
import torch

from _helpers import bits
from oracle import page_fill as pf

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def d():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2609_32663_amd as lib
    return lib


def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEV, dtype=dtype)


class Extend:
    """dkv_page_extend on device copies of a host state."""

    def __init__(self, d, new, length, stack, table, R, Hkv, max_tokens, entries=None, n_entries=None, in_place=True,
                 free_cap=None, n_free=None):
        self.N, self.args = len(length), (R, Hkv)
        free_cap = len(stack) + 2 if free_cap is None else free_cap
        self.d, self.in_place = d, in_place
        self.new, self.length = _dev(new), _dev(length)
        self.stack = _dev(np.concatenate([stack, np.full(free_cap - len(stack), 77)]))
        self.n_free = _dev([len(stack) if n_free is None else n_free])
        self.table = _dev(table)
        self.tok_off = _dev(np.full(self.N + 1, -9))
        self.first_pos = _dev(np.full(self.N, -9))
        self.slots = _dev(np.full((max_tokens, Hkv), -9), torch.int64)
        self.new_len = self.length if in_place else _dev(np.full(self.N, -9))
        self.n_free_out = self.n_free if in_place else _dev([-9])
        self.entries = None if entries is None else _dev(entries)
        self.n_entries = None if n_entries is None else _dev(n_entries)
        self.needed = _dev([-9], torch.int64)
        self.ws = torch.full((d.dkv_page_extend_workspace_bytes(self.N),), 0xA5, dtype=torch.uint8, device=DEV)

    def run(self):
        out = {} if self.in_place else dict(new_len=self.new_len, n_free_out=self.n_free_out)
        self.d.dkv_page_extend(self.new, self.length, self.stack, self.n_free, self.table, *self.args, self.tok_off,
                               self.first_pos, self.slots, self.ws, entries=self.entries, n_entries=self.n_entries,
                               pages_needed=self.needed, **out)
        return self

    def check(self, want):
        torch.cuda.synchronize()
        for name in ("tok_off", "first_pos", "new_len", "table", "slots", "entries", "n_entries"):
            got = getattr(self, name)
            if got is not None:
                np.testing.assert_array_equal(got.cpu().numpy(), want[name], err_msg=name)
        assert int(self.needed) == want["needed"] and int(self.n_free_out) == len(want["stack"])


def _state(rng, N, Hkv, R, longest, spare):
    """Lengths, a table that holds them and the stack of the other pages."""
    length = rng.integers(0, longest + 1, size=N)
    length[rng.uniform(size=N) < 0.3] = 0
    pps = -(-longest // R) + spare
    table = np.full((N * Hkv, pps), -1, dtype=np.int32)
    has = np.arange(pps)[None, :] < np.repeat(-(-length // R), Hkv)[:, None]
    pool = rng.permutation(int(has.sum()) + N * Hkv * spare + 5)
    table[has] = pool[:has.sum()]
    return length, table, pool[has.sum():]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("N,Hkv,R,longest", [(1, 1, 32, 0), (1, 8, 128, 100), (7, 2, 64, 500), (33, 4, 32, 97),
                                             (257, 3, 1024, 5000), (1030, 2, 256, 700), (2100, 1, 512, 40)])
def test_extend_random(d, N, Hkv, R, longest, in_place):
    """Units that get nothing, one token, some and many; entries and counts kept alongside."""
    rng = np.random.default_rng([N, R, in_place])
    length, table, stack = _state(rng, N, Hkv, R, longest, 3)
    new = rng.choice([0, 1, 2, R - 1, R, R + 1, 2 * R], size=N)
    entries = rng.integers(0, 9, size=(N * Hkv, table.shape[1], 4))
    counts = rng.integers(0, 9, size=N * Hkv)
    most = int(new.sum()) + 13  # 13 padded rows
    want = pf.page_extend(new, length, stack.tolist(), table, R, Hkv, most, entries, counts)
    Extend(d, new, length, stack, table, R, Hkv, most, entries, counts, in_place).run().check(want)


@pytest.mark.parametrize("free", [0, 1, 5, 20])
def test_extend_refuses_units(d, free):
    """Too few pages, lengths below zero, tables and token rows that are too short; entries cut at max_entries, or
    none at all."""
    rng = np.random.default_rng(free)
    N, Hkv, R = 12, 2, 32
    length = np.array([0, 31, 32, 5, -1, 64, 90, 0, 96, 95, 10, 0])
    new = np.array([33, 1, 1, -4, 5, 32, 7, 0, 1, 1, 3, 70])
    table = rng.integers(100, 200, size=(N * Hkv, 3))
    table[21, 0] = -1  # a page that is missing: no slot, an entry that names none
    stack = rng.permutation(100)[:free]
    for most in (sum(new[new > 0]), sum(new[new > 0]) - 1, 40, 0):
        entries, counts = np.full((N * Hkv, 2, 4), -3), np.full(N * Hkv, -3)
        want = pf.page_extend(new, length, stack.tolist(), table, R, Hkv, most, entries, counts)
        Extend(d, new, length, stack, table, R, Hkv, most, entries, counts).run().check(want)
        want["entries"] = want["n_entries"] = None
        Extend(d, new, length, stack, table, R, Hkv, most).run().check(want)
    want = pf.page_extend(new, length, [], table, R, Hkv, 200)
    Extend(d, new, length, stack, table, R, Hkv, 200, n_free=-5, in_place=False).run().check(want)
    want = pf.page_extend(new, length, stack.tolist(), table, R, Hkv, 200)  # a height above the stack's room
    Extend(d, new, length, stack, table, R, Hkv, 200, n_free=1000, free_cap=free, in_place=False).run().check(want)


def test_extend_without_units_and_without_tokens(d):
    want = pf.page_extend([], [], [3, 4], np.zeros((0, 3)), 64, 2, 5)
    Extend(d, np.zeros(0), np.zeros(0), np.array([3, 4]), np.zeros((0, 3)), 64, 2, 5).run().check(want)
    table = np.full((4, 2), 6)
    want = pf.page_extend([0, 0], [64, 3], [3, 4], table, 64, 2, 0)
    Extend(d, [0, 0], [64, 3], np.array([3, 4]), table, 64, 2, 0).run().check(want)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("R,long", [(32, 20000), (1024, 40000), (64, 1000), (128, 7900)])
def test_extend_one_long_prompt_among_many_units(d, R, long, in_place):
    """Most rows belong to one unit; the others have none or one."""
    rng = np.random.default_rng(R)
    N, Hkv = 300, 4
    length, table, stack = _state(rng, N, Hkv, R, long, 1 + long // R)
    new = (rng.uniform(size=N) < 0.5).astype(np.int64)
    length[177], new[177] = 0, long
    want = pf.page_extend(new, length, stack.tolist(), table, R, Hkv, int(new.sum()))
    Extend(d, new, length, stack, table, R, Hkv, int(new.sum()), in_place=in_place).run().check(want)


@pytest.mark.parametrize("nseg,pps", [(1, 1), (3, 7), (64, 33), (5, 1024), (300, 100), (4100, 1030)])
@pytest.mark.parametrize("kept", [None, 0.0, 0.4, 1.0])
def test_release_random(d, nseg, pps, kept):
    rng = np.random.default_rng([nseg, pps])
    table = rng.permutation(nseg * pps + 3)[:nseg * pps].reshape(nseg, pps) + 0
    table[rng.uniform(size=table.shape) < 0.2] = -1
    keep = None if kept is None else ((rng.uniform(size=table.shape) < kept) * rng.integers(1, 256, size=table.shape))
    stack = [7, 8, 9]
    for cap in (nseg * pps + 10, 3 + nseg * pps // 3):
        if nseg * pps < 1 << 20:
            want, left = pf.page_release(table, keep, stack, cap)
        else:  # the same, without a Python loop over millions of words
            gone = (table >= 0) & ((keep == 0) if keep is not None else True)
            gone &= (np.cumsum(gone).reshape(gone.shape) <= cap - 3)
            want, left = np.where(gone, -1, table), stack + table[gone].tolist()
        for in_place in (True, False):
            t, n = _dev(table), _dev([3])
            s = _dev(np.concatenate([stack, np.full(cap - 3, -9)]))
            ws = torch.full((d.dkv_page_release_workspace_bytes(nseg, pps),), 0x5A, dtype=torch.uint8, device=DEV)
            to, no = (None, None) if in_place else (torch.full_like(t, -9), torch.full_like(n, -9))
            d.dkv_page_release(t, s, n, ws, keep=None if keep is None else _dev(keep, torch.uint8), table_out=to,
                               n_free_out=no)
            np.testing.assert_array_equal((t if in_place else to).cpu().numpy(), want)
            assert int(n if in_place else no) == len(left)
            np.testing.assert_array_equal(s.cpu().numpy(), left + [-9] * (cap - len(left)))


def test_release_of_no_segments_keeps_the_height(d):
    n, out = _dev([4]), _dev([-1])
    ws = torch.empty(d.dkv_page_release_workspace_bytes(0, 5), dtype=torch.uint8, device=DEV)
    d.dkv_page_release(torch.zeros((0, 5), dtype=torch.int32, device=DEV), _dev(np.arange(9)), n, ws, n_free_out=out)
    assert int(out) == 4


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens,Hkv,R", [(1, 1, 32), (3, 2, 64), (100, 5, 1024), (700, 8, 128)])
def test_append_rows(d, dtype, dim, tokens, Hkv, R):
    """Contiguous rows and parts of wider ones; slots outside the pools are skipped, all other rows stay."""
    rng = np.random.default_rng([dim, tokens])
    pages = -(-tokens * Hkv * 2 // R)
    rand = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dtype)  # noqa: E731
    k, v, x = rand(pages, R, dim), rand(pages, R, dim), rand(tokens, 3 + 2 * Hkv, dim)
    slots = rng.permutation(pages * R)[:tokens * Hkv].reshape(tokens, Hkv)
    slots[rng.uniform(size=slots.shape) < 0.2] = rng.choice([-1, pages * R, 1 << 40, -(1 << 40)])
    kn, vn = x[:, 1:1 + Hkv], x[:, 2 + Hkv:2 + 2 * Hkv]
    want = pf.append_rows(bits(k), bits(v), bits(kn), bits(vn), slots)
    fused = x.to(DEV)
    views = fused[:, 1:1 + Hkv], fused[:, 2 + Hkv:2 + 2 * Hkv]
    for kd, vd in (views, (views[0].contiguous(), views[1].contiguous())):
        kp, vp = k.to(DEV), v.to(DEV)
        d.dkv_paged_append(kd, vd, _dev(slots, torch.int64), kp, vp)
        np.testing.assert_array_equal(bits(kp), want[0])
        np.testing.assert_array_equal(bits(vp), want[1])


def test_append_past_2_31_elements(d):
    """Slots whose byte offsets pass 32 bits, in pools of 9 GiB."""
    R, dim, pages = 1024, 128, 36865
    k = torch.empty((pages, R, dim), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    at = torch.tensor([[0], [1 << 23], [1 << 24], [(1 << 25) + 7], [pages * R - 1]], device=DEV)
    x = torch.randn((5, 2, dim), device=DEV).to(torch.bfloat16)
    d.dkv_paged_append(x[:, :1], x[:, 1:], at, k, v)
    assert torch.equal(k.view(-1, dim)[at[:, 0]], x[:, 0]) and torch.equal(v.view(-1, dim)[at[:, 0]], x[:, 1])


def test_requests_come_grow_and_go(d):
    """Several steps in place on one state: requests are admitted, grow by single tokens and chunks, and finish; the
    pages of finished ones are handed out again.  The second half replays captured calls."""
    rng = np.random.default_rng(11)
    N, Hkv, R, pps, most = 6, 2, 32, 8, 400
    free = rng.permutation(40)
    table, length = np.full((N * Hkv, pps), -1), np.zeros(N, dtype=np.int64)
    x = Extend(d, np.zeros(N), length, free, table, R, Hkv, most, np.zeros((N * Hkv, pps, 4)), np.zeros(N * Hkv),
               free_cap=40)
    keep = torch.ones((N * Hkv, pps), dtype=torch.uint8, device=DEV)
    rws = torch.empty(d.dkv_page_release_workspace_bytes(N * Hkv, pps), dtype=torch.uint8, device=DEV)
    stack, entries, counts = free.tolist(), np.zeros((N * Hkv, pps, 4)), np.zeros(N * Hkv)
    graph = None

    def step():
        d.dkv_page_release(x.table, x.stack, x.n_free, rws, keep=keep)
        x.run()

    for i in range(12):
        new = rng.choice([0, 1, 1, 40, 90], size=N)
        done = rng.uniform(size=N) < 0.25
        length[done] = 0
        host_keep = np.repeat(~done, Hkv)[:, None].repeat(pps, 1).astype(np.uint8)
        table, stack = pf.page_release(table, host_keep, stack, 40)
        want = pf.page_extend(new, length, stack, table, R, Hkv, most, entries, counts)
        keep.copy_(_dev(host_keep, torch.uint8))
        x.new.copy_(_dev(new))
        x.length.copy_(_dev(length))
        if i < 6:
            step()
        else:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step()
            graph.replay()
        x.check(want)
        table, stack, entries, counts = want["table"], want["stack"], want["entries"], want["n_entries"]
        length = want["new_len"].astype(np.int64)
        np.testing.assert_array_equal(x.stack.cpu().numpy()[:len(stack)], stack)


def test_pools_that_are_parameters(d):
    """A subclass of Tensor is a tensor."""
    pool = torch.nn.Parameter(torch.zeros((3, 32, 64), device=DEV), requires_grad=False)
    other = torch.nn.Parameter(torch.zeros((3, 32, 64), device=DEV), requires_grad=False)
    x = torch.nn.Parameter(torch.ones((2, 1, 64), device=DEV), requires_grad=False)
    d.dkv_paged_append(x, x, _dev([[5], [70]], torch.int64), pool, other)
    for p in (pool, other):
        assert p.view(96, 64)[[5, 70]].eq(1).all() and float(p.sum()) == 128.0
