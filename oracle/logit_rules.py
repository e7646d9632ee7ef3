"""Rules on logits, row by row and token by token, in 64 bits."""
import numpy as np


def path_of(parent, node):
    out = []
    while node >= 0:
        out.append(int(node))
        node = parent[node]
    return out[::-1]


def process(logits, rows, tree_prompt, tree_off, parent, token, hist=None, hist_off=None, prompt_len=None, repetition=None,
            frequency=None, presence=None, temperature=None, bias=None, mask=None, mask_row=None):
    """logits [R,V]; rows: their nodes; bias: per prompt a list of (token, value); mask [n,V] truth values.  Returns (out,
    sum of the sizes of what was added up, for the roundings)."""
    z = np.array(logits, dtype=np.float64)
    size = np.abs(z)
    for r, node in enumerate(rows):
        t = int(np.searchsorted(tree_off, node, side="right")) - 1
        p = int(tree_prompt[t])
        text = [] if hist_off is None or hist is None else [int(x) for x in hist[hist_off[t]:hist_off[t + 1]]]
        text += [int(token[n]) for n in path_of(parent, node)]
        made = text[(0 if prompt_len is None else max(0, int(prompt_len[t]))):]
        if repetition is not None:
            for v in set(text):
                z[r, v] = z[r, v] / repetition[p] if z[r, v] > 0 else z[r, v] * repetition[p]
                size[r, v] = max(size[r, v], abs(z[r, v]))
        for v in set(made):
            f = (0 if frequency is None else frequency[p] * made.count(v)) + (0 if presence is None else presence[p])
            z[r, v] -= f
            size[r, v] += abs(f) + (0 if frequency is None else abs(frequency[p]) * made.count(v))
        if bias is not None:
            for v, b in dict(bias[p]).items():
                z[r, v] += b
                size[r, v] += abs(b)
        if temperature is not None:
            z[r] /= temperature[p]
            size[r] /= temperature[p]
        m = -1 if mask is None else r if mask_row is None else int(mask_row[r])
        if m >= 0:
            z[r, ~mask[m]] = -np.inf
    return z, size
