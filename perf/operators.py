"""The operators of a paged cache that is filled on the GPU, as a serving program
calls them, and the same computed by elementary torch operations.

A server admits requests, cuts their prompts into chunks and runs the chunks
of some requests and single tokens of the others in one batch.  Per batch it
extends the page tables (extend), writes the new K and V rows into their slots
(append) and lets every new token attend to what its request holds (attend); a
compressed or finished request gives its pages back (release).  A case's
"kind" is one of

  extend   dkv_page_extend: tables, slots, token offsets and entries from lengths
  release  dkv_page_release: the pages that a selection, or a finished request, leaves
  append   dkv_paged_append: rows of K and V into their slots
  attend   dkv_paged_query_attn: a chunk of every sequence over its pages
  step     extend, append and attend of one batch, in a row

Shapes are those of 8B and Qwen-shaped attention layers and a small test
model; requests hold from nothing to 128K tokens.  q, K and V are Gaussian,
tables are shuffled.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
SCRATCH = 512 << 20  # bytes of scratch that the server keeps for its attention calls


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _case(kind, name=None, **kw):
    # context: positions of the longest request before the call; chunk: most new tokens of a request;
    # new: "all" requests bring chunk tokens, "ragged" 1 to chunk, "mixed" some chunk and the others one;
    # retained: share of the context that a selection kept (1.0: whole pages)
    c = {"kind": kind, "dtype": "bf16", "layers": 1, "batch": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page_rows": 128, "context": 0, "chunk": 1, "new": "all", "ragged": False, "retained": 1.0, "fused": True}
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest step there is: three tokens of one short request of the small test model
        _case("step", "step_tiny", q_heads=4, kv_heads=2, head_dim=64, page_rows=32, context=100, chunk=3),
        # a decode step of 32 requests of 2K to 16K tokens, one 8B layer: reading the cache bounds it
        _case("step", "step_8b_decode_bs32", batch=32, context=16384, ragged=True),
        # two prompt chunks among 31 single tokens, Qwen-shaped layer (7 query heads a KV head), small pages
        _case("step", "step_qwen_mixed_bs33", batch=33, q_heads=28, kv_heads=4, page_rows=64, context=4097, chunk=1000,
              new="mixed", ragged=True),
        # one chunk of a long prompt: 512 tokens after 32K, one 8B layer
        _case("attend", "attend_8b_chunk_512_32k", context=32768, chunk=512, page_rows=256),
        # two prompts from their first token, up to 4K, one 8B layer: the heaviest arithmetic
        _case("attend", "attend_8b_prompts_4k", batch=2, chunk=4096, new="ragged"),
        # a long question to a compressed 128K context (whole and partial pages kept), one 8B layer
        _case("attend", "attend_8b_question_128k", context=131072, chunk=256, retained=0.346),
        # a decode step's tables for 64 requests on all 32 layers: most tokens find room in the last page
        _case("extend", "extend_8b_decode_bs64", layers=32, batch=64, context=8192, ragged=True),
        # four prompts of up to 8K tokens admitted on all 32 layers
        _case("extend", "extend_8b_admit_8k", layers=32, batch=4, chunk=8192, new="ragged"),
        # one layer of one finished 4K request
        _case("release", "release_4k_request", context=4100, retained=0.0),
        # all 32 layers of a 128K context after a selection that kept 35%
        _case("release", "release_8b_stack_128k", layers=32, context=131072, retained=0.346),
        # single tokens of 96 requests, Qwen-shaped, fp32
        _case("append", "append_qwen_bs96_f32", dtype="f32", batch=96, q_heads=28, kv_heads=4, page_rows=64,
              context=4097, ragged=True),
        # a batch of 8K new tokens, one 8B layer, K and V as parts of the fused projection's rows
        _case("append", "append_8b_8k_tokens", batch=8, context=2049, chunk=1024, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 8), (32, 8), (64, 8), (28, 4), (28, 4), (4, 2), (16, 16), (12, 4), (32, 2), (40, 8)]


def draw(rng):
    kind = rng.choice(["extend", "release", "append", "attend", "attend", "attend", "attend", "step", "step", "step"])
    q, kv = rng.choice(_HEADS)
    c = _case(kind, q_heads=q, kv_heads=kv, head_dim=rng.choice([128, 128, 128, 64]),
              page_rows=rng.choice([32, 64, 128, 128, 256, 512, 1024]), fused=rng.random() < 0.7)
    c["context"] = rng.choice([0, _log_int(rng, 1, 131072), _log_int(rng, 256, 32768)])
    c["chunk"] = rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 16, 4096)])
    c["batch"] = _log_int(rng, 1, 64)
    c["new"] = rng.choice(["all", "ragged", "mixed"])
    c["ragged"] = rng.random() < 0.6
    if kind in ("extend", "release"):
        c["layers"] = _log_int(rng, 1, 32)
    if kind == "append":
        c["dtype"] = rng.choice(["bf16", "f32"])
    if kind == "attend" and c["context"] >= 4096 and rng.random() < 0.5:
        c["retained"], c["ragged"], c["new"] = round(rng.uniform(0.15, 0.6), 3), False, "all"
    if kind == "release":
        c["retained"], c["ragged"] = rng.choice([0.0, round(rng.uniform(0.1, 0.9), 3)]), False
        c["context"] = max(1, c["context"])
    # no dearer than the dearest listed case that has this kind's work, and a cache of at most 8M rows
    like = [work(x) for x in listed() if (x["kind"] in ("attend", "step")) == (kind in ("attend", "step"))]
    most = {m: max(w[m] for w in like) for m in ("bytes", "flops")}
    while True:
        w = work(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and (
                c["batch"] * kv * (c["context"] + c["chunk"]) <= 1 << 23):
            return c
        k = max(("batch", "layers", "chunk", "context"), key=lambda x: (c[x] > 1, c[x] ** (2 if x == "chunk" else 1)))
        c[k] = max(1, c[k] // 2)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _lengths(c):
    """Positions held before the call and new tokens, of every request; the case alone decides them."""
    rng = np.random.default_rng([c["batch"], c["context"], c["chunk"]])
    B = c["batch"]
    held = np.full(B, c["context"], dtype=np.int64)
    if c["ragged"] and c["context"] > 0:
        held = rng.integers(c["context"] // 8, c["context"] + 1, size=B)
        held[rng.integers(B)] = c["context"]
    new = np.full(B, c["chunk"], dtype=np.int64)
    if c["new"] == "ragged":
        new = rng.integers(1 + c["chunk"] // 8, c["chunk"] + 1, size=B)
        new[rng.integers(B)] = c["chunk"]
    if c["new"] == "mixed":
        new = np.ones(B, dtype=np.int64)
        new[rng.permutation(B)[:max(1, B // 16)]] = c["chunk"]
    return held, new


def _kept(c, rng, T):
    """bool [T]: sink, recent window and a run of every retained stretch of 32 to 1,024 positions."""
    n = rng.integers(32, 1025, size=T // 32 + 1)
    edge = np.minimum(np.cumsum(n), T)
    keep = np.repeat(rng.random(n.size) < c["retained"], np.diff(np.concatenate([[0], edge])))
    if c["retained"] > 0:
        keep[:128] = True
        keep[max(0, T - 512):] = True
    return keep


def _pages(c, held, seed):
    """Page table int32 [segments][pages] with `held` positions of every segment paged, -1 elsewhere; the stack of
    the other pages, and the pool's size."""
    rows = c["page_rows"]
    _, new = _lengths(c)
    per_seg = np.repeat(np.tile(held, c["layers"]), c["kv_heads"])
    grown = np.repeat(np.tile(held + new, c["layers"]), c["kv_heads"])
    pps = int(-(-(c["context"] + c["chunk"]) // rows)) + 1
    count, room = -(-per_seg // rows), -(-grown // rows)
    total = int(np.maximum(count, room).sum()) + 3
    perm = np.random.default_rng([seed, total]).permutation(total).astype(np.int32)
    table = np.full((per_seg.size, pps), -1, dtype=np.int32)
    has = np.arange(pps)[None, :] < count[:, None]
    table[has] = perm[:int(count.sum())]
    return table, perm[int(count.sum()):].copy(), total


def _entries(table, lengths, rows):
    """Entries int32 [segments][pages][4] of whole pages (page, logical page, first slot, past the last), and counts."""
    nseg, pps = table.shape
    at = np.arange(pps)
    e = np.zeros((nseg, pps, 4), dtype=np.int32)
    count = -(-lengths // rows)
    has = at[None, :] < count[:, None]
    e[..., 0] = np.where(has, table, 0)
    e[..., 1] = np.where(has, at[None, :], 0)
    e[..., 3] = np.clip(lengths[:, None] - at[None, :] * rows, 0, rows)
    return e, count.astype(np.int32)


def _selected(c, table, seed):
    """Entries of a selection: every maximal run of kept positions within a page, then the appended tokens' pages."""
    rows, T, new = c["page_rows"], c["context"], c["chunk"]
    found, kept = [], []
    for s in range(table.shape[0]):
        keep = _kept(c, np.random.default_rng([seed, s]), T)
        pos = np.flatnonzero(keep)
        starts = np.flatnonzero(np.concatenate([[True], (np.diff(pos) != 1) | (pos[1:] % rows == 0)]))
        lo = pos[starts]
        hi = pos[np.concatenate([starts[1:], [pos.size]]) - 1] + 1
        at = np.arange(T, T + new)
        tlo = at[(at == T) | (at % rows == 0)]
        lo, hi = np.concatenate([lo, tlo]), np.concatenate([hi, np.append(tlo[1:], T + new)])
        page = lo // rows
        found.append(np.stack([table[s][page], page, lo - page * rows, hi - page * rows], axis=1))
        kept.append(pos)
    most = max(len(f) for f in found)
    e = np.zeros((len(found), most, 4), dtype=np.int32)
    for s, f in enumerate(found):
        e[s, :len(f)] = f
    return e, np.array([len(f) for f in found], dtype=np.int32), kept


def _int(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEV, dtype=dtype)


def _randn(shape, gen, c):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)


def prepare(case, seed):
    c = dict(case)
    held, new = _lengths(c)
    L, B, Hq, Hkv, dim, rows = c["layers"], c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page_rows"]
    N, S = L * B, L * B * Hkv
    tokens = int(new.sum())
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    st = {"c": c, "N": N, "tokens": tokens, "max_q": int(new.max()), "scale": 1.0 / math.sqrt(dim)}
    before = held if c["kind"] in ("extend", "step") else held + new
    table, free, num_pages = _pages(c, before, seed)
    st["table"] = _int(table)
    st["num_pages"] = num_pages
    if c["kind"] == "release":
        keep = np.zeros(table.shape, dtype=np.uint8)
        if c["retained"] > 0:
            rng = np.random.default_rng(seed)
            keep = (rng.random(table.shape) < c["retained"]).astype(np.uint8)
        st.update(keep=_int(keep, torch.uint8), table_out=torch.zeros_like(st["table"]), n_free_out=_int([0]),
                  stack=_int(np.concatenate([free, np.full(num_pages - free.size, -7)])), n_free=_int([free.size]),
                  ws=torch.empty(8 * S + 4096, dtype=torch.uint8, device=DEV))
        return st
    if c["kind"] in ("extend", "step"):
        e, count = _entries(table, np.repeat(np.tile(held, L), Hkv), rows)
        st.update(unit_len=_int(np.tile(held, L)), unit_new=_int(np.tile(new, L)), stack=_int(free),
                  n_free=_int([free.size]), n_free_out=_int([0]), new_len=torch.zeros(N, dtype=torch.int32, device=DEV),
                  tok_off=torch.zeros(N + 1, dtype=torch.int32, device=DEV),
                  first_pos=torch.zeros(N, dtype=torch.int32, device=DEV),
                  slots=torch.zeros((L * tokens, Hkv), dtype=torch.int64, device=DEV),
                  entries=_int(e), n_entries=_int(count), needed=torch.zeros(1, dtype=torch.int64, device=DEV),
                  ews=torch.empty(64 * N + 4096, dtype=torch.uint8, device=DEV))
    else:
        off = np.concatenate([[0], np.cumsum(new)])
        st.update(tok_off=_int(off), first_pos=_int(held))
        if c["kind"] == "append":
            seq = np.repeat(np.arange(B), new)
            pos = held[seq] + np.arange(tokens) - off[seq]
            seg = seq[:, None] * Hkv + np.arange(Hkv)[None, :]
            st["slots"] = _int(table[seg, (pos // rows)[:, None]].astype(np.int64) * rows + (pos % rows)[:, None],
                               torch.int64)
        elif c["retained"] < 1.0:
            e, count, st["kept"] = _selected(c, table, seed)
            st.update(entries=_int(e), n_entries=_int(count))
        else:
            e, count = _entries(table, np.repeat(held + new, Hkv), rows)
            st.update(entries=_int(e), n_entries=_int(count))
    if c["kind"] == "extend":
        return st
    # the batch's projections, token-major: parts of one fused buffer's rows, or tensors of their own
    if c["fused"]:
        x = _randn((tokens, Hq + 2 * Hkv, dim), gen, c)
        st.update(q=x[:, :Hq], k_new=x[:, Hq:Hq + Hkv], v_new=x[:, Hq + Hkv:])
    else:
        st.update(q=_randn((tokens, Hq, dim), gen, c), k_new=_randn((tokens, Hkv, dim), gen, c),
                  v_new=_randn((tokens, Hkv, dim), gen, c))
    st.update(k=_randn((num_pages, rows, dim), gen, c), v=_randn((num_pages, rows, dim), gen, c))
    if c["kind"] in ("attend", "step"):
        if "kept" in st:  # the host knows the lengths: what a program hands over as the expected rows
            st["rows"] = int(st["n_entries"].sum()) * rows
        else:
            st["rows"] = int((-(-(held + new) // rows) * rows).sum()) * Hkv
        st["most"] = [int(-(-n // rows)) for n in held + new] if "kept" not in st else [int(st["n_entries"].max())] * B
        st["offsets"] = np.concatenate([[0], np.cumsum(new)]).tolist()
        st["out"] = torch.zeros((tokens, Hq, dim), dtype=torch.float32, device=DEV)
        st["ws"] = torch.empty(SCRATCH, dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _extend(st):
    c = st["c"]
    if own:
        import paper_2609_32663_amd as d
        d.dkv_page_extend(st["unit_new"], st["unit_len"], st["stack"], st["n_free"], st["table"], c["page_rows"],
                          c["kv_heads"], st["tok_off"], st["first_pos"], st["slots"], st["ews"], new_len=st["new_len"],
                          n_free_out=st["n_free_out"], entries=st["entries"], n_entries=st["n_entries"],
                          pages_needed=st["needed"])
        return
    rows, Hkv, N = c["page_rows"], c["kv_heads"], st["N"]
    table, (nseg, pps) = st["table"], st["table"].shape
    length, new = st["unit_len"].long(), st["unit_new"].long()
    grown = length + new
    end = torch.cumsum(new.clamp(min=0), 0)
    start = end - new.clamp(min=0)
    room = st["slots"].shape[0]
    valid = (length >= 0) & (new >= 0) & (grown <= pps * rows) & (end <= room)
    first_page, page_end = (length + rows - 1) // rows, (grown + rows - 1) // rows
    per = torch.where(valid, page_end - first_page, 0)  # of one segment
    base = torch.cumsum(per * Hkv, 0) - per * Hkv
    served = valid & ((base + per * Hkv <= st["n_free"]) | (per == 0))
    st["needed"].copy_((per * Hkv).sum())
    st["n_free_out"].copy_(st["n_free"] - torch.where(served, per * Hkv, 0).sum())
    st["tok_off"][0].zero_()
    st["tok_off"][1:].copy_(end.clamp(max=room))
    st["first_pos"].copy_(torch.where(served, length, -1))
    st["new_len"].copy_(torch.where(served, grown, length))
    # new pages, from the top of the stack: segment by segment, page by page
    at = torch.arange(pps, device=DEV)[None, None, :]
    g = torch.arange(Hkv, device=DEV)[None, :, None]
    rank = base[:, None, None] + g * per[:, None, None] + at - first_page[:, None, None]
    mine = served[:, None, None] & (at >= first_page[:, None, None]) & (at < page_end[:, None, None])
    top = st["n_free"].long() - 1
    page = st["stack"][(top - rank).clamp(min=0, max=max(0, st["stack"].shape[0] - 1))] if st["stack"].numel() else rank
    table.copy_(torch.where(mine, page.int(), table.view(N, Hkv, pps)).view(nseg, pps))
    # slots of the new tokens
    t = torch.arange(room, device=DEV)
    u = torch.searchsorted(end, t, right=True).clamp(max=N - 1)
    pos = length[u] + t - start[u]
    owner = u[:, None] * Hkv + torch.arange(Hkv, device=DEV)[None, :]
    p = table[owner, (pos // rows).clamp(min=0, max=pps - 1)[:, None]].long()
    ok = (served[u] & (t < end[-1]))[:, None] & (p >= 0)
    st["slots"].copy_(torch.where(ok, p * rows + (pos % rows)[:, None], -1))
    # entries of the pages that changed
    touched = served[:, None, None] & (new > 0)[:, None, None] & (at >= (length // rows)[:, None, None]) & (
        at < page_end[:, None, None])
    e = st["entries"].view(N, Hkv, -1, 4)
    hi = (grown[:, None, None] - at * rows).clamp(min=0, max=rows).expand(N, Hkv, pps)
    fresh = torch.stack([table.view(N, Hkv, pps), at.int().expand(N, Hkv, pps), torch.zeros_like(hi).int(), hi.int()], -1)
    e.copy_(torch.where(touched[..., None], fresh, e))
    count = st["n_entries"].view(N, Hkv)
    count.copy_(torch.where(served[:, None], page_end[:, None].int(), count))


def _release(st):
    if own:
        import paper_2609_32663_amd as d
        d.dkv_page_release(st["table"], st["stack"], st["n_free"], st["ws"], keep=st["keep"], table_out=st["table_out"],
                           n_free_out=st["n_free_out"])
        return
    table = st["table"].view(-1)
    gone = (table >= 0) & (st["keep"].view(-1) == 0)
    rank = torch.cumsum(gone, 0) - 1
    st["table_out"].view(-1).copy_(torch.where(gone, -1, table))
    # the released pages go behind the stack's, in table order; the others to a place past its end
    to = torch.where(gone, st["n_free"].long() + rank, st["stack"].shape[0])
    wide = torch.cat([st["stack"], table[:1]])
    st["stack"].copy_(wide.scatter(0, to, table)[:-1])
    st["n_free_out"].copy_(st["n_free"] + gone.sum())


def _append(st):
    if own:
        import paper_2609_32663_amd as d
        d.dkv_paged_append(st["k_new"], st["v_new"], st["slots"], st["k"], st["v"])
        return
    dim = st["c"]["head_dim"]
    at = st["slots"].reshape(-1)
    st["k"].view(-1, dim).index_copy_(0, at, st["k_new"].reshape(-1, dim))
    st["v"].view(-1, dim).index_copy_(0, at, st["v_new"].reshape(-1, dim))


def _attend(st):
    c = st["c"]
    if own:
        import paper_2609_32663_amd as d
        d.dkv_paged_query_attn(st["q"], st["tok_off"], st["first_pos"], st["k"], st["v"], st["entries"],
                               st["n_entries"], st["scale"], st["out"], st["ws"], c["kv_heads"], st["max_q"],
                               rows_hint=st["rows"])
        return
    Hkv, G, dim, rows = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"], c["page_rows"]
    slot = torch.arange(rows, device=DEV, dtype=torch.int32)
    for b in range(c["batch"]):  # sequences of other lengths; all the heads of one at once
        lo, hi, n = st["offsets"][b], st["offsets"][b + 1], st["most"][b]
        m = hi - lo
        e = st["entries"][b * Hkv:(b + 1) * Hkv, :n]
        listed_ = torch.arange(n, device=DEV)[None, :] < st["n_entries"][b * Hkv:(b + 1) * Hkv, None]
        named = (slot >= e[..., 2:3]) & (slot < e[..., 3:4]) & listed_[..., None]
        pos = torch.where(named, e[..., 1:2] * rows + slot, 1 << 30).view(Hkv, 1, n * rows)
        k = st["k"][e[..., 0].long()].view(Hkv, n * rows, dim).float()
        v = st["v"][e[..., 0].long()].view(Hkv, n * rows, dim).float()
        q = st["q"][lo:hi].reshape(m, Hkv, G, dim).transpose(0, 1).reshape(Hkv, m * G, dim).float()
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * st["scale"]
        own_pos = st["first_pos"][b] + torch.arange(m, device=DEV).repeat_interleave(G, output_size=m * G)
        s.masked_fill_(pos > own_pos[None, :, None], -math.inf)
        s -= s.amax(dim=2, keepdim=True)
        s.exp_()
        o = torch.matmul(s, v) / s.sum(dim=2, keepdim=True)
        st["out"][lo:hi] = o.view(Hkv, m, G, dim).transpose(0, 1).reshape(m, Hkv * G, dim)


def run(st):
    kind = st["c"]["kind"]
    if kind == "release":
        _release(st)
        return {"table": st["table_out"], "stack": st["stack"], "n_free": st["n_free_out"]}
    if kind == "append":
        _append(st)
        return {"k": st["k"], "v": st["v"]}
    if kind == "attend":
        _attend(st)
        return st["out"]
    _extend(st)
    got = {"new_len": st["new_len"], "tok_off": st["tok_off"], "first_pos": st["first_pos"], "table": st["table"],
           "slots": st["slots"], "entries": st["entries"], "n_entries": st["n_entries"], "n_free": st["n_free_out"],
           "needed": st["needed"]}
    if kind == "step":
        _append(st)
        _attend(st)
        got.update(k=st["k"], v=st["v"], out=st["out"])
    return got


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it computes
# ---------------------------------------------------------------------------

def work(case):
    c = case
    held, new = _lengths(c)
    e = 2 if c["dtype"] == "bf16" else 4
    L, Hq, Hkv, dim, rows = c["layers"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page_rows"]
    tokens = int(new.sum())
    total = {"bytes": 0, "flops": 0}
    if c["kind"] in ("extend", "step"):
        # a slot per token and head; table word, stack word and entry of each new page; per segment a page read, an
        # entry and a count written; per request the lengths
        pages = int((-(-(held + new) // rows) - -(-held // rows)).sum())
        total["bytes"] += L * (tokens * Hkv * 8 + Hkv * pages * 24 + c["batch"] * (Hkv * 24 + 20))
    if c["kind"] in ("append", "step"):
        total["bytes"] += tokens * Hkv * (4 * dim * e + 8)
    if c["kind"] in ("attend", "step"):
        seen = (held * c["retained"] + new).sum() * Hkv
        pairs = ((held * c["retained"]) * new + new * (new + 1) / 2).sum() * Hq
        total["bytes"] += int(seen * (2 * dim * e + 16 / rows)) + tokens * Hq * dim * (e + 4)
        total["flops"] += int(4 * dim * pairs)
    if c["kind"] == "release":
        # the table and the marks read, the table written; a word per released page
        words = L * c["batch"] * Hkv * (int(-(-(c["context"] + c["chunk"]) // rows)) + 1)
        total["bytes"] += int(words * (9 + 4 * (1 - c["retained"])))
    return total


def exact(case, seed):
    """Attention in 64 bits from the page table and the positions; everything else is copied or whole numbers."""
    c = case
    if c["kind"] not in ("attend", "step"):
        return None
    st = prepare(case, seed)
    f = torch.float64
    Hkv, G, dim, rows = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"], c["page_rows"]
    held, new = _lengths(c)
    out = torch.zeros((st["tokens"], c["q_heads"], dim), dtype=f, device=DEV)
    k_rows, v_rows = st["k"].view(-1, dim), st["v"].view(-1, dim)
    table = st["table"].long()
    at = 0
    for b, (h, n) in enumerate(zip(held.tolist(), new.tolist())):
        for g in range(Hkv):
            s = b * Hkv + g
            kept = torch.arange(h, device=DEV)
            if "kept" in st:
                kept = torch.from_numpy(st["kept"][s]).to(DEV)
            here = torch.arange(h, h + n, device=DEV)
            if c["kind"] == "step":  # the new tokens are not in the cache yet
                src = table[s][kept // rows] * rows + kept % rows
                k = torch.cat([k_rows[src], st["k_new"][at:at + n, g]]).to(f)
                v = torch.cat([v_rows[src], st["v_new"][at:at + n, g]]).to(f)
            else:
                pos = torch.cat([kept, here])
                src = table[s][pos // rows] * rows + pos % rows
                k, v = k_rows[src].to(f), v_rows[src].to(f)
            pos = torch.cat([kept, here])
            kt = k.t().contiguous()
            for i in range(0, n, 512):
                m = min(512, n - i)
                q = st["q"][at + i:at + i + m, g * G:(g + 1) * G].reshape(m * G, dim).to(f)
                z = torch.mm(q, kt) * st["scale"]
                mine = here[i:i + m].repeat_interleave(G)
                z.masked_fill_(pos[None, :] > mine[:, None], -math.inf)
                out[at + i:at + i + m, g * G:(g + 1) * G] = torch.mm(torch.softmax(z, dim=1), v).view(m, G, dim)
        at += n
    if c["kind"] == "attend":
        return out
    names = ("new_len", "tok_off", "first_pos", "table", "slots", "entries", "n_entries", "n_free", "needed", "k", "v")
    return {**dict.fromkeys(names), "out": out}
