"""Rotary positions, rows of a cache in 8 bits, drafted trees and attention over
them, step by step in NumPy and float64.  Nothing here comes from the paper: it
is the bookkeeping of a server that speculates, and the definitions of the
formats that its cache is kept in."""

import numpy as np

__all__ = ["rope", "codes_to_values", "quantise", "row_values", "tree_plan", "accept", "tree_attn"]


def rope(x, pos, inv_freq, rot_dim, interleaved=False, mscale=1.0):
    """x [tokens][heads][dim] float64 turned pair by pair; a token with a negative position is left as it is."""
    out = np.array(x, dtype=np.float64, copy=True)
    n = rot_dim // 2
    for t in range(out.shape[0]):
        if pos[t] < 0:
            continue
        for i in range(n):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
            angle = float(pos[t]) * float(inv_freq[i])
            c, s = np.cos(angle), np.sin(angle)
            xa, xb = np.array(x[t, :, a], np.float64), np.array(x[t, :, b], np.float64)
            out[t, :, a] = mscale * (xa * c - xb * s)
            out[t, :, b] = mscale * (xa * s + xb * c)
    return out


def codes_to_values(codes):
    """Values of e4m3 codes (uint8): sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    c = np.asarray(codes, dtype=np.int64)
    ex, man = (c >> 3) & 15, c & 7
    v = np.where(ex > 0, (1 + man / 8.0) * 2.0 ** (ex - 7.0), man / 8.0 * 2.0 ** -6)
    v = np.where((c & 0x7F) == 0x7F, np.nan, v)
    return np.where(c & 0x80, -v, v)


_LADDER = codes_to_values(np.arange(127))           # the non-negative finite values, ascending
_BORDERS = (_LADDER[:-1] + _LADDER[1:]) / 2.0


def quantise(x):
    """Rows [..., d] (float64) as (codes uint8 [..., d], exponent bytes uint8 [...])."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    most = np.where(finite, np.abs(x), 0.0).max(axis=-1)
    e = np.full(most.shape, -60, dtype=np.int64)
    while True:  # the smallest exponent that is large enough
        small = (most > 448.0 * 2.0 ** e) & (e < 120)
        if not small.any():
            break
        e[small] += 1
    y = np.where(finite, x, 0.0) * 2.0 ** -e[..., None].astype(np.float64)
    size = np.minimum(np.abs(y), np.where(e == 120, 240.0, 448.0)[..., None])
    at = np.searchsorted(_BORDERS, size, side="left")   # a value on a border goes to the lower code ...
    tie = (at < len(_BORDERS)) & (_BORDERS[np.minimum(at, len(_BORDERS) - 1)] == size) & (at % 2 == 1)
    code = at + tie                                     # ... unless the upper one is the even
    code = np.where(finite, code | np.where(np.signbit(x), 0x80, 0), 0x7F)
    return code.astype(np.uint8), (e + 127).astype(np.uint8)


def row_values(codes, exponents):
    return codes_to_values(codes) * 2.0 ** (np.asarray(exponents, np.float64) - 127.0)[..., None]


def tree_plan(tok_off, first_pos, max_q, num_tokens, parent=None, words=0):
    """Positions int32 [tokens] and ancestor bits uint64 [tokens][words]."""
    pos = np.full(num_tokens, -1, dtype=np.int64)
    mask = np.zeros((num_tokens, words), dtype=np.uint64)
    for b in range(len(first_pos)):
        lo, hi = min(int(tok_off[b]), num_tokens), min(int(tok_off[b + 1]), num_tokens)
        if first_pos[b] < 0:
            continue
        for t in range(min(hi - lo, max_q)):
            a, depth = t, -1
            while a >= 0:
                depth += 1
                if words:
                    mask[lo + t, a // 64] |= np.uint64(1 << (a % 64))
                up = a - 1 if parent is None else int(parent[lo + a])
                a = up if up < a else -1
            pos[lo + t] = min(int(first_pos[b]) + depth, 2 ** 31 - 2)
    return pos, mask


def accept(first_pos, path, n_path, table, page_rows, num_kv_heads, pools):
    """pools: arrays [num_pages][page_rows][...] whose rows move.  Returns the new pools, new_len (None for units that
    are left out) and keep."""
    pools = [np.array(x, copy=True) for x in pools]
    pages = pools[0].shape[0]
    B, R, pps = len(path), page_rows, table.shape[1]
    new_len, keep = [], np.full(table.shape, -1, dtype=np.int64)
    for n in range(len(first_pos)):
        first, b = int(first_pos[n]), n % B
        if first < 0:
            new_len.append(None)
            continue
        line = []
        for x in path[b][:max(0, int(n_path[b]))].tolist():
            if x < 0 or (line and x <= line[-1]) or first + x >= pps * R or first + x >= 2 ** 31 - 1:
                break
            line.append(x)
        new_len.append(first + len(line))
        for g in range(num_kv_heads):
            s = n * num_kv_heads + g
            keep[s] = np.arange(pps) < -(-new_len[-1] // R)
            for i, x in enumerate(line):
                src, dst = int(table[s, (first + x) // R]), int(table[s, (first + i) // R])
                if x != i and 0 <= src < pages and 0 <= dst < pages:
                    for pool in pools:
                        pool[dst, (first + i) % R] = pool[src, (first + x) % R]
    return pools, new_len, keep


def tree_attn(q, tok_off, first_pos, k_rows, v_rows, page_rows, entries, n_entries, sm_scale, num_kv_heads, max_q,
              mask=None):
    """Attention of every new token to the positions below its sequence's first new one and to the new tokens j whose
    bit it has (no mask: those up to itself).  q [tokens][Hq][d], k_rows, v_rows [pages][page_rows][d]: float64 values.
    Zeros where nothing is seen; NaN in rows that no sequence owns."""
    rows, Hq, d = q.shape
    pages, R, G = k_rows.shape[0], page_rows, Hq // num_kv_heads
    out = np.full((rows, Hq, d), np.nan)
    for b in range(len(first_pos)):
        lo, hi = int(tok_off[b]), min(int(tok_off[b + 1]), int(tok_off[b]) + max_q, rows)
        out[lo:hi] = 0.0
        first = int(first_pos[b])
        if first < 0:
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
            known = pos < first + hi - lo
            page, slot, j = page[known], slot[known], pos[known] - first
            kr, vr = k_rows[page, slot], v_rows[page, slot]
            for t in range(lo, hi):
                if mask is None:
                    see = j <= t - lo
                else:
                    bits = np.unpackbits(np.ascontiguousarray(mask[t]).view(np.uint8), bitorder="little")
                    own = np.zeros(len(j), dtype=bool)
                    new = (j >= 0) & (j < len(bits))
                    own[new] = bits[j[new]] != 0
                    see = (j < 0) | own
                if not see.any():
                    continue
                sc = sm_scale * (q[t, g * G:(g + 1) * G] @ kr[see].T)
                p = np.exp(sc - sc.max(axis=1, keepdims=True))
                out[t, g * G:(g + 1) * G] = (p @ vr[see]) / p.sum(axis=1, keepdims=True)
    return out
