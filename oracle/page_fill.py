"""Filling a paged cache and attending a chunk over it, step by step in plain
Python and float64.  Nothing here comes from the paper: it is the bookkeeping
of a server whose requests grow in pages, and causal attention over them."""

import numpy as np

from .dkv_oracle import widen

__all__ = ["page_extend", "page_release", "append_rows", "chunk_attn"]


def page_extend(unit_new, unit_len, stack, page_table, page_rows, num_kv_heads, max_tokens, entries=None,
                n_entries=None):
    """Gives every unit the pages for its new tokens, unit by unit.

    stack: list of free pages, the top at the end.  entries: int32
    [N * Hkv][max_entries][4], n_entries int32 [N * Hkv], or None.  Returns a
    dict of new arrays (and the stack left)."""
    N, Hkv, R = len(unit_len), int(num_kv_heads), int(page_rows)
    table = np.array(page_table, copy=True)
    stack = list(stack)
    new_len = np.array(unit_len, dtype=np.int32, copy=True)
    first_pos = np.full(N, -1, dtype=np.int32)
    tok_off = [0]
    slots = np.full((max_tokens, Hkv), -1, dtype=np.int64)
    entries = None if entries is None else np.array(entries, copy=True)
    n_entries = None if n_entries is None else np.array(n_entries, copy=True)
    needed, height = 0, len(stack)
    for n in range(N):
        have, add = int(unit_len[n]), int(unit_new[n])
        row = tok_off[-1]
        tok_off.append(row + max(add, 0))
        if have < 0 or add < 0 or have + add > min(table.shape[1] * R, 2 ** 31 - 1) or tok_off[-1] > max_tokens:
            continue
        old, grown = -(-have // R), -(-(have + add) // R)
        needed += Hkv * (grown - old)
        if grown > old and needed > height:
            continue
        first_pos[n] = have
        new_len[n] = have + add
        for g in range(Hkv):
            s = n * Hkv + g
            for p in range(old, grown):
                table[s, p] = stack.pop()
            for t in range(add):
                pos = have + t
                page = int(table[s, pos // R])
                if page >= 0:
                    slots[row + t, g] = page * R + pos % R
                if entries is not None and pos // R < entries.shape[1]:
                    entries[s, pos // R] = (page, pos // R, 0, min(R, have + add - pos // R * R))
            if n_entries is not None and add > 0:
                n_entries[s] = grown
    return dict(table=table, stack=stack, new_len=new_len, first_pos=first_pos,
                tok_off=np.minimum(tok_off, max_tokens).astype(np.int32), slots=slots, entries=entries,
                n_entries=n_entries, needed=needed)


def page_release(page_table, keep, stack, free_cap):
    """Pushes the pages that `keep` (None: none of them) does not mark; returns the table and the stack left."""
    table, stack = np.array(page_table, copy=True), list(stack)
    for s in range(table.shape[0]):
        for p in range(table.shape[1]):
            if table[s, p] >= 0 and (keep is None or keep[s, p] == 0) and len(stack) < free_cap:
                stack.append(int(table[s, p]))
                table[s, p] = -1
    return table, stack


def append_rows(k_pages, v_pages, k_new, v_new, slots):
    """New tokens' rows [tokens][Hkv][d] into pool rows slots[t][g]; slots outside the pools are skipped."""
    out = []
    for pool, new in ((k_pages, k_new), (v_pages, v_new)):
        flat = np.array(pool, copy=True).reshape(-1, pool.shape[-1])
        for t in range(slots.shape[0]):
            for g in range(slots.shape[1]):
                if 0 <= slots[t, g] < flat.shape[0]:
                    flat[slots[t, g]] = new[t, g]
        out.append(flat.reshape(pool.shape))
    return out


def chunk_attn(q, tok_off, first_pos, k_pages, v_pages, entries, n_entries, sm_scale, num_kv_heads, dtype, max_q):
    """Attention of token i of sequence b, at position first_pos[b] + i, to the slots of its segment's entries at or
    below that position; zeros for a sequence with a negative first_pos and for a token that sees nothing.  Float64
    [tokens][Hq][d]; NaN in rows that no sequence owns."""
    qf = widen(q, dtype)
    rows, Hq, d = qf.shape
    R, pages = k_pages.shape[1], k_pages.shape[0]
    G = Hq // num_kv_heads
    out = np.full((rows, Hq, d), np.nan)
    for b in range(len(first_pos)):
        lo, hi = int(tok_off[b]), min(int(tok_off[b + 1]), int(tok_off[b]) + max_q)
        out[lo:hi] = 0.0
        if first_pos[b] < 0:
            continue
        for g in range(num_kv_heads):
            s = b * num_kv_heads + g
            where = []
            for page, lp, a, z in np.asarray(entries[s])[:max(0, int(n_entries[s]))].tolist():
                if 0 <= page < pages and 0 <= a and z <= R and lp >= 0:
                    where += [(page, slot, lp * R + slot) for slot in range(a, z)]
            if not where:
                continue
            page, slot, pos = np.array(where).T
            limit = int(first_pos[b]) + hi - lo
            page, slot, pos = page[pos < limit], slot[pos < limit], pos[pos < limit]
            kr, vr = widen(k_pages[page, slot], dtype), widen(v_pages[page, slot], dtype)
            for t in range(lo, hi):
                see = pos <= int(first_pos[b]) + t - lo
                if not see.any():
                    continue
                sc = sm_scale * (qf[t, g * G:(g + 1) * G] @ kr[see].T)
                p = np.exp(sc - sc.max(axis=1, keepdims=True))
                out[t, g * G:(g + 1) * G] = (p @ vr[see]) / p.sum(axis=1, keepdims=True)
    return out
