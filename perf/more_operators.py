"""The operators of speculative decoding over a quantised paged cache, as a serving program calls them, and the same
computed by elementary torch operations.

A server drafts a tree of tokens for every request.  It rotates the queries and keys by their positions, writes K and
V into the paged cache in 8 bits (store), lets every drafted token attend to what its request holds and to its own
ancestors (attend), and keeps the accepted path (accept).  Prompts in chunks and single tokens take the same calls
without a tree.  A case's "kind" is one of

  rope     dkv_rope: rotary positions of token-major rows
  store    dkv_paged_store, then dkv_paged_load of the same rows: rotation, quantised write, and reading it back
  load     dkv_paged_load: rows of a quantised context read back
  attend   dkv_paged_tree_attn: a chunk, or a tree of drafted tokens, of every sequence over its pages
  step     dkv_tree_plan, store, attend and dkv_paged_accept of one batch in a row, then the batch's rows as the cache
           holds them (dkv_paged_load)

The cache is "f8" (rows of e4m3 with a power of two per row) or "bf16".  Shapes are those of 8B and Qwen-shaped
attention layers and a small test model; requests hold from nothing to 128K tokens.  Some channels of K are larger
than others, as after training; page tables are shuffled.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
SCRATCH = 512 << 20  # bytes of scratch that the server keeps for its attention calls
F8 = torch.float8_e4m3fn


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _case(kind, name=None, **kw):
    # context: positions of the longest request before the call; chunk: most new tokens of a request;
    # new: "all" requests bring chunk tokens, "ragged" 1 to chunk, "mixed" some chunk and the others one;
    # tree: new tokens are a drafted tree (each has a parent among the ones before it), else a chain;
    # rot: rotated part of a head; scaled: how the frequencies are stretched for long contexts
    c = {"kind": kind, "cache": "f8", "dtype": "bf16", "batch": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "page_rows": 128, "context": 0, "chunk": 1, "new": "all", "ragged": False, "tree": False, "fused": True,
         "rot": 128, "interleaved": False, "scaled": "wave"}
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # three tokens of the small test model
        _case("rope", "rope_tiny", q_heads=4, kv_heads=2, head_dim=64, rot=64, context=100, chunk=3, scaled="plain"),
        # a batch of 8K tokens of prompts, one 8B layer, q and k as parts of the fused projection's rows
        _case("rope", "rope_8b_8k_tokens", batch=8, context=16384, chunk=1024),
        # part of a head, pairs next to each other, an odd number of tokens, fp32
        _case("rope", "rope_part_pairs_f32", dtype="f32", q_heads=20, kv_heads=20, head_dim=96, rot=40, context=5000,
              chunk=1001, interleaved=True, scaled="linear"),
        # single tokens of 96 requests, Qwen-shaped
        _case("store", "store_qwen_bs96", batch=96, q_heads=28, kv_heads=4, page_rows=64, context=4097, ragged=True,
              scaled="plain"),
        # a batch of 8K new tokens, one 8B layer
        _case("store", "store_8b_8k_tokens", batch=8, context=2049, chunk=1024, ragged=True),
        # a short request's rows
        _case("load", "load_qwen_900", q_heads=28, kv_heads=4, page_rows=64, chunk=900),
        # a whole context of 128K tokens, one 8B layer
        _case("load", "load_8b_128k", chunk=131072, page_rows=256),
        # a decode step of 32 requests of 2K to 16K tokens, one 8B layer: reading the cache bounds it
        _case("attend", "attend_8b_decode_bs32", batch=32, context=16384, ragged=True),
        # one chunk of a long prompt, 512 tokens after 32K, one 8B layer: the heaviest arithmetic
        _case("attend", "attend_8b_chunk_512_32k", context=32768, chunk=512, page_rows=256),
        # trees of 48 drafted tokens for 8 requests of up to 32K tokens, 64 query heads
        _case("attend", "attend_tree_48_bs8", batch=8, q_heads=64, context=32768, chunk=48, ragged=True, tree=True),
        # the smallest step there is: a tree of five tokens of one short request of the small test model
        _case("step", "step_tiny_tree", q_heads=4, kv_heads=2, head_dim=64, rot=64, page_rows=32, context=100, chunk=5,
              tree=True, scaled="plain"),
        # trees of up to 24 drafted tokens for 16 requests of up to 16K tokens, one 8B layer
        _case("step", "step_8b_tree_bs16", batch=16, context=16384, chunk=24, new="ragged", ragged=True, tree=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 8), (32, 8), (64, 8), (28, 4), (28, 4), (4, 2), (16, 16), (12, 4), (32, 2), (40, 8)]


def draw(rng):
    kind = rng.choice(["rope", "rope", "store", "store", "load", "attend", "attend", "attend", "attend", "step", "step"])
    q, kv = rng.choice(_HEADS)
    dim = rng.choice([128, 128, 128, 64])
    c = _case(kind, q_heads=q, kv_heads=kv, head_dim=dim, page_rows=rng.choice([32, 64, 128, 128, 256, 512, 1024]),
              fused=rng.random() < 0.7, cache=rng.choice(["f8", "f8", "f8", "bf16"]),
              interleaved=rng.random() < 0.4, scaled=rng.choice(["plain", "linear", "wave", "ramp"]))
    if kind == "rope":
        c["head_dim"] = dim = rng.choice([64, 80, 96, 128, 128, 256])
        c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    c["rot"] = rng.choice([dim, dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)])
    c["context"] = rng.choice([0, _log_int(rng, 1, 131072), _log_int(rng, 256, 32768)])
    c["chunk"] = rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 2, 64), _log_int(rng, 16, 4096)])
    c["batch"] = _log_int(rng, 1, 64)
    c["new"] = rng.choice(["all", "ragged", "mixed"])
    c["ragged"] = rng.random() < 0.6
    c["tree"] = kind == "step" or rng.random() < 0.5
    if c["tree"]:
        c["chunk"] = min(c["chunk"], 512)
    if kind == "load":
        c["context"], c["chunk"] = 0, _log_int(rng, 1, 131072)
    # no dearer than the dearest listed case that has this kind's work, a cache of at most 4M rows, and a bounded
    # number of scores
    like = [work(x) for x in listed() if (x["kind"] in ("attend", "step")) == (kind in ("attend", "step"))]
    most = {m: max(w[m] for w in like) for m in ("bytes", "flops")}
    while True:
        w, rows = work(c), c["context"] + c["chunk"]
        scores = c["batch"] * q * c["chunk"] * rows if kind in ("attend", "step") else 0
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and c["batch"] * kv * rows <= 1 << 22 and (
                scores <= 1 << 30):
            return c
        k = max(("batch", "chunk", "context"), key=lambda x: (c[x] > 1, c[x] ** (2 if x == "chunk" else 1)))
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


def _frequencies(c):
    """Angle per position of every rotated pair, fp32: plain, all divided by a factor (linear), or divided by it where
    the wave is long, by its wavelength (wave) or by the pair's place (ramp)."""
    n, base, factor, first = c["rot"] // 2, 500000.0, 8.0, 8192.0
    f = base ** (-np.arange(n, dtype=np.float64) / n)
    if c["scaled"] == "linear":
        f = f / factor
    if c["scaled"] == "wave":
        smooth = np.clip((first * f / (2 * math.pi) - 1.0) / 3.0, 0.0, 1.0)
        f = (1 - smooth) * f / factor + smooth * f
    if c["scaled"] == "ramp":
        lo, hi = (n * math.log(first / (2 * math.pi * t)) / math.log(base) for t in (32.0, 1.0))
        ramp = np.clip((np.arange(n) - math.floor(lo)) / max(1.0, math.ceil(hi) - math.floor(lo)), 0.0, 1.0)
        f = f / factor * ramp + f * (1 - ramp)
    return f.astype(np.float32)


def _pages(c, held, seed):
    """Page table int32 [segments][pages] of `held` positions of every request, shuffled, and the pool's size."""
    rows, Hkv = c["page_rows"], c["kv_heads"]
    count = np.repeat(-(-held // rows), Hkv)
    pps = int(count.max()) + 1
    total = int(count.sum()) + 3
    table = np.full((count.size, pps), -1, dtype=np.int32)
    table[np.arange(pps)[None, :] < count[:, None]] = np.random.default_rng([seed, total]).permutation(total)[:total - 3]
    return table, total


def _entries(table, lengths, rows):
    """Entries int32 [segments][pages][4] of whole pages (page, logical page, first slot, past the last), and counts."""
    at = np.arange(table.shape[1])
    e = np.zeros((*table.shape, 4), dtype=np.int32)
    count = -(-lengths // rows)
    has = at[None, :] < count[:, None]
    e[..., 0] = np.where(has, table, 0)
    e[..., 1] = np.where(has, at[None, :], 0)
    e[..., 3] = np.clip(lengths[:, None] - at[None, :] * rows, 0, rows)
    return e, count.astype(np.int32)


def _trees(new, seed):
    """Parents (index among a request's new tokens, -1: the last token it held), ancestors as bits of int64 words
    [tokens][words], and an accepted path of every request (-1 past its end) with its length."""
    rng = np.random.default_rng([seed, 77])
    words = -(-int(new.max()) // 64)
    parents, masks, paths = [], [], []
    for n in new.tolist():
        i = np.arange(n)
        p = rng.integers(np.maximum(-1, i - 9), i)
        bits = np.zeros((n, words * 64), dtype=np.uint8)
        for t in range(n):
            if p[t] >= 0:
                bits[t] = bits[p[t]]
            bits[t, t] = 1
        line = np.flatnonzero(bits[rng.integers(n)])
        parents.append(p)
        masks.append(np.packbits(bits, axis=1, bitorder="little").view(np.int64))
        paths.append(line[:rng.integers(0, min(16, line.size) + 1)])
    path = np.full((len(paths), 16), -1, dtype=np.int32)
    for i, x in enumerate(paths):
        path[i, :x.size] = x
    return np.concatenate(parents), np.concatenate(masks), path, np.array([x.size for x in paths])


def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEV, dtype=dtype)


def prepare(case, seed):
    c = dict(case)
    held, new = _lengths(c)
    B, Hq, Hkv, dim, rows = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["page_rows"]
    tokens = int(new.sum())
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    kind, dtype = c["kind"], torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    off = np.concatenate([[0], np.cumsum(new)])
    seq = np.repeat(np.arange(B), new)
    here = np.arange(tokens) - off[seq]  # index among the request's new tokens
    st = {"c": c, "tokens": tokens, "max_q": int(new.max()), "scale": 1.0 / math.sqrt(dim), "tok_off": _dev(off),
          "first_pos": _dev(held), "freq": _dev(_frequencies(c), torch.float32), "mscale": 1.0}
    if c["scaled"] == "ramp":
        st["mscale"] = 0.1 * math.log(8.0) + 1.0
    past = here  # how far a new token's position is past the request's
    if c["tree"]:
        parent, mask, path, n_path = _trees(new, seed)
        past = np.unpackbits(mask.view(np.uint8), axis=1).sum(axis=1, dtype=np.int64) - 1
    st["pos"] = _dev(held[seq] + past)
    # the batch's projections, token-major: parts of one fused buffer's rows, or tensors of their own; of K every
    # sixteenth channel is six times as large
    wide = torch.ones(dim, device=DEV)
    wide[::16] = 6.0
    x = torch.randn((tokens, Hq + 2 * Hkv, dim), generator=gen, device=DEV)
    x[:, Hq:Hq + Hkv] *= wide
    x = x.to(dtype)
    if kind == "rope":
        x = x if c["fused"] else x[:, :Hq + Hkv].contiguous()
        st.update(x=x[:, :Hq + Hkv], out=torch.zeros((tokens, Hq + Hkv, dim), dtype=dtype, device=DEV))
        return st
    split = [x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]]
    st["q"], st["k_new"], st["v_new"] = split if c["fused"] else [y.contiguous() for y in split]
    # the cache: rows as the server has written them earlier
    table, num_pages = _pages(c, held + new, seed)
    k = torch.randn((num_pages, rows, dim), generator=gen, device=DEV).mul_(wide)
    v = torch.randn((num_pages, rows, dim), generator=gen, device=DEV)
    if c["cache"] == "f8":
        (st["k"], ke), (st["v"], ve) = _quantise(k), _quantise(v)
        st["scales"] = torch.stack([ke, ve], dim=-1)
    else:
        st.update(k=k.bfloat16(), v=v.bfloat16(), scales=None)
    del k, v
    at = held[seq] + here
    segment = seq[:, None] * Hkv + np.arange(Hkv)[None, :]
    st["slots"] = _dev(table[segment, (at // rows)[:, None]].astype(np.int64) * rows + (at % rows)[:, None], torch.int64)
    st["table"] = _dev(table)
    if kind in ("store", "load", "step"):
        st.update(q_out=torch.zeros((tokens, Hq, dim), dtype=dtype, device=DEV),
                  k_out=torch.zeros((tokens, Hkv, dim), dtype=dtype, device=DEV),
                  v_out=torch.zeros((tokens, Hkv, dim), dtype=dtype, device=DEV))
    if kind in ("attend", "step"):
        e, count = _entries(table, np.repeat(held + new, Hkv), rows)
        st.update(entries=_dev(e), n_entries=_dev(count), rows=int((-(-(held + new) // rows) * rows).sum()) * Hkv,
                  mask=_dev(mask, torch.int64) if c["tree"] else None,
                  out=torch.zeros((tokens, Hq, dim), dtype=torch.float32, device=DEV),
                  ws=torch.empty(SCRATCH, dtype=torch.uint8, device=DEV))
    if kind == "step":
        st.update(parent=_dev(parent), path=_dev(path), n_path=_dev(n_path), made=torch.zeros_like(st["mask"]),
                  made_pos=torch.zeros_like(st["pos"]), new_len=torch.zeros_like(st["first_pos"]),
                  keep=torch.zeros(table.shape, dtype=torch.uint8, device=DEV))
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _quantise(x):
    """Rows of e4m3 and the exponent byte (127 + e) of each row's power of two: the smallest that holds the row's
    largest value below 448."""
    x = x.float()
    bits = x.abs().amax(dim=-1).view(torch.int32)
    e = ((bits >> 23) - 135 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(-117, 120)
    y = x * ((127 - e) << 23).view(torch.float32)[..., None]
    most = torch.where(e == 120, 240.0, 448.0)[..., None]
    return torch.minimum(torch.maximum(y, -most), most).to(F8), (e + 127).to(torch.uint8)


def _values(rows, exponents):
    """fp32 values of rows of the cache."""
    if rows.dtype is not F8:
        return rows.float()
    return rows.float() * (exponents.int() << 23).view(torch.float32)[..., None]


def _rotated(st, x, pos):
    """x [tokens][heads][dim] rotated by its positions, angles and products in 64 bits."""
    c, n = st["c"], st["c"]["rot"] // 2
    angle = pos.double()[:, None] * st["freq"].double()[None, :]
    cos, sin = (angle.cos() * st["mscale"])[:, None], (angle.sin() * st["mscale"])[:, None]
    y = x.double()
    a, b = (y[..., 0:2 * n:2], y[..., 1:2 * n:2]) if c["interleaved"] else (y[..., :n], y[..., n:2 * n])
    u, w = a * cos - b * sin, a * sin + b * cos
    both = torch.stack([u, w], dim=-1).flatten(-2) if c["interleaved"] else torch.cat([u, w], dim=-1)
    return torch.cat([both, y[..., 2 * n:]], dim=-1).float()


def _plain_store(st, pos):
    dim, at = st["c"]["head_dim"], st["slots"].view(-1)
    st["q_out"].copy_(_rotated(st, st["q"], pos))
    k = _rotated(st, st["k_new"], pos).view(-1, dim)
    v = st["v_new"].reshape(-1, dim)
    if st["scales"] is None:
        st["k"].view(-1, dim)[at] = k.bfloat16()
        st["v"].view(-1, dim)[at] = v
        return
    (k, ke), (v, ve) = _quantise(k), _quantise(v)
    st["k"].view(torch.uint8).view(-1, dim)[at] = k.view(torch.uint8)
    st["v"].view(torch.uint8).view(-1, dim)[at] = v.view(torch.uint8)
    st["scales"].view(-1, 2)[at] = torch.stack([ke, ve], dim=-1)


def _rows_at(st, at):
    """fp32 K and V of pool rows `at`."""
    dim, exps = st["c"]["head_dim"], None if st["scales"] is None else st["scales"].view(-1, 2)[at]
    got = []
    got.append(_values(_pick(st["k"], dim, at), None if exps is None else exps[..., 0]))
    got.append(_values(_pick(st["v"], dim, at), None if exps is None else exps[..., 1]))
    return got


def _pick(pool, dim, at):
    if pool.dtype is F8:
        return pool.view(torch.uint8).view(-1, dim)[at].view(F8)
    return pool.view(-1, dim)[at]


def _plain_load(st):
    k, v = _rows_at(st, st["slots"])
    st["k_out"].copy_(k)
    st["v_out"].copy_(v)


def _padded(st):
    """Index [B][most new tokens] of every request's tokens in the token-major arrays, and which of them exist."""
    i = torch.arange(st["max_q"], device=DEV)
    at = st["tok_off"][:-1, None] + i
    return at.clamp(max=st["tokens"] - 1).long(), at < st["tok_off"][1:, None]


def _plain_attend(st, q, mask):
    c = st["c"]
    B, Hkv, G, dim, rows = c["batch"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"], c["page_rows"]
    n, S = st["max_q"], st["entries"].shape[1] * rows
    token, real = _padded(st)
    slot = torch.arange(rows, device=DEV)
    e = st["entries"].long()
    listed_ = torch.arange(e.shape[1], device=DEV)[None, :] < st["n_entries"][:, None]
    named = (slot >= e[..., 2:3]) & (slot < e[..., 3:4]) & listed_[..., None]
    k, v = _rows_at(st, (e[..., 0:1] * rows + slot).view(B, Hkv, S))
    # key j of the new tokens, or below zero for what the request held
    j = torch.where(named, e[..., 1:2] * rows + slot, 1 << 30).view(B, Hkv, 1, S) - st["first_pos"].view(B, 1, 1, 1)
    i = torch.arange(n, device=DEV)
    if mask is None:
        sees = j <= i.view(1, 1, n, 1)
    else:
        bits = (mask[token][..., None] >> torch.arange(64, device=DEV) & 1).view(B, 1, n, -1).bool()
        column = j.clamp(0, bits.shape[-1] - 1).expand(B, Hkv, n, S)
        sees = (j < 0) | (bits.expand(B, Hkv, n, -1).gather(3, column) & (j < st["max_q"]))
    x = q[token].float().view(B, n, Hkv, G, dim).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, dim)
    s = torch.matmul(x, k.transpose(2, 3).contiguous()).view(B, Hkv, n, G, S) * st["scale"]
    s.masked_fill_(~sees[:, :, :, None], -math.inf)
    s -= s.amax(dim=-1, keepdim=True)
    s.exp_()
    total = s.sum(dim=-1, keepdim=True)
    o = torch.matmul(s.view(B, Hkv, n * G, S), v).view(B, Hkv, n, G, dim) / total
    st["out"][token[real]] = o.permute(0, 2, 1, 3, 4).reshape(B, n, Hkv * G, dim)[real]


def _plain_plan(st):
    """Ancestors of every drafted token as bits, and its position: by how many links it hangs below the last one."""
    B, n = st["c"]["batch"], st["max_q"]
    token, real = _padded(st)
    parent = torch.where(real, st["parent"][token], -1).long()
    # a place behind the tokens is its own parent; the links' reach doubles
    hop = torch.cat([torch.where(parent >= 0, parent, n), torch.full((B, 1), n, device=DEV)], dim=1)
    sees = torch.zeros((B, n + 1, n + 1), dtype=torch.bool, device=DEV)
    sees.diagonal(dim1=1, dim2=2)[:, :n] = True
    links = 1
    while links <= n:
        sees = sees | sees.gather(1, hop[:, :, None].expand_as(sees))
        hop = hop.gather(1, hop)
        links *= 2
    seen = sees[:, :n, :n]
    st["made_pos"][token[real]] = (st["first_pos"][:, None] + seen.sum(dim=2) - 1).int()[real]
    words = st["made"].shape[1]
    wide = torch.zeros((B, n, words * 64), dtype=torch.int64, device=DEV)
    wide[..., :n] = seen
    bits = (wide.view(B, n, words, 64) << torch.arange(64, device=DEV)).sum(dim=3)
    st["made"][token[real]] = bits[real]


def _plain_accept(st):
    c = st["c"]
    B, Hkv, dim, rows = c["batch"], c["kv_heads"], c["head_dim"], c["page_rows"]
    pps, n = st["table"].shape[1], st["path"].shape[1]
    i = torch.arange(n, device=DEV)
    takes = i < st["n_path"][:, None]
    table = st["table"].view(B, Hkv, pps).long()

    def row_of(pos):
        page = table.gather(2, (pos // rows).clamp(max=pps - 1)[:, None].expand(B, Hkv, n))
        return page * rows + (pos % rows)[:, None]

    first = st["first_pos"].long()[:, None]
    move = takes[:, None].expand(B, Hkv, n)
    src, dst = row_of(first + st["path"].clamp(min=0))[move], row_of(first + i)[move]
    wide = st["k"].dtype is F8
    for name in ("k", "v"):
        pool = (st[name].view(torch.uint8) if wide else st[name]).view(-1, dim)
        pool[dst] = pool[src]
    if wide:
        st["scales"].view(-1, 2)[dst] = st["scales"].view(-1, 2)[src]
    st["new_len"].copy_(st["first_pos"] + st["n_path"])
    pages = (st["new_len"] + rows - 1) // rows
    st["keep"].copy_((torch.arange(pps, device=DEV) < pages[:, None]).repeat_interleave(Hkv, dim=0))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _store(st, pos):
    if own:
        import paper_2609_32663_amd as d
        d.dkv_paged_store(st["k_new"], st["v_new"], st["slots"], st["k"], st["v"], scales=st["scales"], q=st["q"],
                          q_out=st["q_out"], pos=pos, inv_freq=st["freq"], rot_dim=st["c"]["rot"],
                          interleaved=st["c"]["interleaved"], mscale=st["mscale"])
    else:
        _plain_store(st, pos)


def _load(st):
    if own:
        import paper_2609_32663_amd as d
        d.dkv_paged_load(st["slots"], st["k"], st["v"], st["k_out"], st["v_out"], scales=st["scales"])
    else:
        _plain_load(st)


def _attend(st, q, mask):
    if own:
        import paper_2609_32663_amd as d
        d.dkv_paged_tree_attn(q, st["tok_off"], st["first_pos"], st["k"], st["v"], st["entries"], st["n_entries"],
                              st["scale"], st["out"], st["ws"], st["c"]["kv_heads"], st["max_q"], mask=mask,
                              scales=st["scales"], rows_hint=st["rows"])
    else:
        _plain_attend(st, q, mask)


def run(st):
    c = st["c"]
    if c["kind"] == "rope":
        if own:
            import paper_2609_32663_amd as d
            d.dkv_rope(st["x"], st["pos"], st["freq"], c["rot"], st["out"], interleaved=c["interleaved"],
                       mscale=st["mscale"])
        else:
            st["out"].copy_(_rotated(st, st["x"], st["pos"]))
        return st["out"]
    if c["kind"] == "store":
        _store(st, st["pos"])
        _load(st)
        return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}
    if c["kind"] == "load":
        _load(st)
        return {"k": st["k_out"], "v": st["v_out"]}
    if c["kind"] == "attend":
        _attend(st, st["q"], st["mask"])
        return st["out"]
    if own:
        import paper_2609_32663_amd as d
        d.dkv_tree_plan(st["tok_off"], st["first_pos"], st["max_q"], st["made_pos"], parent=st["parent"], mask=st["made"])
    else:
        _plain_plan(st)
    _store(st, st["made_pos"])
    _attend(st, st["q_out"], st["made"])
    if own:
        d.dkv_paged_accept(st["first_pos"], st["path"], st["n_path"], st["table"], c["kv_heads"], st["k"], st["v"],
                           st["new_len"], scales=st["scales"], keep=st["keep"])
    else:
        _plain_accept(st)
    _load(st)
    return {"mask": st["made"], "pos": st["made_pos"], "q": st["q_out"], "out": st["out"], "new_len": st["new_len"],
            "keep": st["keep"], "k": st["k_out"], "v": st["v_out"]}


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it computes
# ---------------------------------------------------------------------------

def work(case):
    c = case
    held, new = _lengths(c)
    e = 2 if c["dtype"] == "bf16" else 4
    Hq, Hkv, dim, rows = c["q_heads"], c["kv_heads"], c["head_dim"], c["page_rows"]
    row = dim + 1 if c["cache"] == "f8" else 2 * dim  # bytes of a row of K or V in the cache
    tokens = int(new.sum())
    total = {"bytes": 0, "flops": 0}
    if c["kind"] == "rope":
        total["bytes"] += tokens * ((Hq + Hkv) * dim * 2 * e + 4) + 2 * c["rot"]
        total["flops"] += 3 * tokens * (Hq + Hkv) * c["rot"]
    if c["kind"] in ("store", "step"):
        # q read and written, K and V read and written in the cache's type, a slot per row
        total["bytes"] += tokens * (4 * Hq * dim + Hkv * (4 * dim + 2 * row + 8))
        total["flops"] += 3 * tokens * (Hq + Hkv) * c["rot"]
    if c["kind"] in ("store", "load", "step"):
        total["bytes"] += tokens * Hkv * (2 * row + 4 * dim + 8)
    if c["kind"] in ("attend", "step"):
        seen = (held + new).sum() * Hkv
        depth = np.minimum((new + 1) / 2, 2 * np.log2(new + 1) + 1) if c["tree"] else (new + 1) / 2  # own tokens seen
        total["bytes"] += int(seen * (2 * row + 16 / rows)) + tokens * Hq * dim * 6
        total["flops"] += int(4 * dim * ((held + depth) * new).sum() * Hq)
    if c["kind"] == "step":
        total["bytes"] += c["batch"] * Hkv * 4 * 4 * row + tokens * 16
    return total


# ---------------------------------------------------------------------------
# results in 64 bits
# ---------------------------------------------------------------------------

def _turned(st, x, pos):
    """Rotation as a product of complex numbers."""
    n = st["c"]["rot"] // 2
    turn = torch.polar(torch.full((st["tokens"], 1, n), st["mscale"], dtype=torch.float64, device=DEV),
                       torch.outer(pos.double(), st["freq"].double())[:, None])
    y = x.double().clone()
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if st["c"]["interleaved"] else (slice(0, n), slice(n, 2 * n))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _as_held(st, x):
    """The values that the cache holds for rows x (64 bits): four significant bits, steps of 2^(e - 9) at least."""
    if st["scales"] is None:
        return x.bfloat16().double()
    most = x.abs().amax(dim=-1, keepdim=True)
    e = torch.ceil(torch.log2(most / 448.0)).clamp(-117, 120)
    y = x * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def _held(st, at):
    """64-bit K and V of pool rows `at`, from their bits."""
    dim = st["c"]["head_dim"]
    if st["scales"] is None:
        return st["k"].view(-1, dim)[at].double(), st["v"].view(-1, dim)[at].double()
    code = np.arange(256)
    size = np.where(code >> 3 & 15, (8 + (code & 7)) * 2.0 ** ((code >> 3 & 15) - 10.0), (code & 7) * 2.0 ** -9)
    value = _dev(np.where(code >> 7, -size, size), torch.float64)
    power = torch.exp2(st["scales"].view(-1, 2)[at].double() - 127)
    k, v = (value[st[x].view(torch.uint8).view(-1, dim)[at].int()] for x in ("k", "v"))
    return k * power[..., 0:1], v * power[..., 1:2]


def exact(case, seed):
    """From the inputs and the page table in 64 bits, one sequence and head at a time."""
    c = case
    st = prepare(case, seed)
    kind, pos = c["kind"], st["pos"]
    if kind == "rope":
        return _turned(st, st["x"], pos)
    if kind == "load":
        k, v = _held(st, st["slots"])
        return {"k": k, "v": v}
    q, fresh = st["q"], None
    if kind != "attend":
        q = _turned(st, q, pos)
        fresh = _as_held(st, _turned(st, st["k_new"], pos).float().double()), _as_held(st, st["v_new"].double())
    if kind == "store":
        return {"q": q, "k": fresh[0], "v": fresh[1]}
    Hkv, G, dim, rows = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"], c["page_rows"]
    held, new = _lengths(c)
    x = q if kind == "attend" else q.bfloat16()
    out = torch.zeros((st["tokens"], c["q_heads"], dim), dtype=torch.float64, device=DEV)
    at = 0
    for b, (h, n) in enumerate(zip(held.tolist(), new.tolist())):
        sees = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()
        if st["mask"] is not None:
            j = torch.arange(n, device=DEV)
            sees = (st["mask"][at:at + n][:, j // 64] >> (j % 64)) & 1 == 1
        for g in range(Hkv):
            p = torch.arange(h if fresh is not None else h + n, device=DEV)
            k, v = _held(st, st["table"][b * Hkv + g].long()[p // rows] * rows + p % rows)
            if fresh is not None:
                k, v = (torch.cat([a, f[at:at + n, g]]) for a, f in zip((k, v), fresh))
            kt = k.t().contiguous()
            for i in range(0, n, 512):
                m = min(512, n - i)
                z = torch.mm(x[at + i:at + i + m, g * G:(g + 1) * G].reshape(m * G, dim).double(), kt) * st["scale"]
                z[:, h:].masked_fill_(~sees[i:i + m].repeat_interleave(G, dim=0), -math.inf)
                out[at + i:at + i + m, g * G:(g + 1) * G] = torch.mm(torch.softmax(z, dim=1), v).view(m, G, dim)
        at += n
    if kind == "attend":
        return out
    # accepted rows move to the front of the request's new ones
    for b, (n, take) in enumerate(zip(st["tok_off"].tolist(), st["n_path"].tolist())):
        line = st["path"][b, :take].long() + n
        for f in fresh:
            f[n:n + take] = f[line].clone()
    return {"mask": None, "pos": None, "q": q, "out": out, "new_len": None, "keep": None, "k": fresh[0], "v": fresh[1]}
