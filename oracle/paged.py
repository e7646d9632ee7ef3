"""A paged cache in plain words: where a token lies, what a row of a chunk sees, its attention in 64 bits."""
import numpy as np


def place(page_table, page_size, s, t):
    """(page, slot) of token t of sequence s, or None behind the table's end."""
    i = t // page_size
    return (int(page_table[s][i]), t % page_size) if i < len(page_table[s]) else None


def gather(pages, page_table, page_size, s, n):
    """Tokens 0 .. n-1 of a sequence as [n,Hkv,D] in 64 bits, and which of them are there; pages [n_pages, page, Hkv, D]."""
    out, there = np.zeros((n,) + pages.shape[2:]), np.zeros(n, dtype=bool)
    for t in range(n):
        at = place(page_table, page_size, s, t)
        if at is not None and 0 <= at[0] < pages.shape[0]:
            out[t], there[t] = pages[at[0], at[1]], True
    return out, there


def attend(q, k, v, there, ctx, scale, anc=None):
    """Rows q [n,Hq,D] of a chunk behind ctx tokens over k, v [ctx+n,Hkv,D].  Returns (out, lse, weights' sum of |v|)."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, lse, size = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf), np.zeros((n, Hq, D))
    for i in range(n):
        sees = there.copy()
        if anc is None:
            sees[ctx + i + 1:] = False
        else:
            sees[ctx:] &= np.array([(int(anc[i]) >> j) & 1 for j in range(len(there) - ctx)], dtype=bool)
        if not sees.any():
            continue
        for h in range(Hq):
            z = k[sees, h // G] @ q[i, h] * scale
            m = z.max()
            p = np.exp(z - m)
            lse[i, h] = m + np.log(p.sum())
            out[i, h], size[i, h] = p @ v[sees, h // G] / p.sum(), p @ np.abs(v[sees, h // G]) / p.sum()
    return out, lse, size
