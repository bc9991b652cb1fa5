"""fp64 definitions of the token operators on NumPy arrays (test infrastructure only).

Each follows the formula directly and shares no code with the library. The gradients that are
sums also come with the sum of the absolute values of their terms: the scale that rounding
errors are bounded by.
"""
import numpy as np


def embed(ids, table, scale):
    out = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids):
        if i >= len(table):
            out[t] = np.nan
        elif i >= 0:
            out[t] = scale * table[i]
    return out


def embed_backward(ids, grad, vocab, scale, into=None):
    """(gradient of the table, scale of its sums, number of terms of each row)."""
    table = np.zeros((vocab, grad.shape[1])) if into is None else into.copy()
    size, terms = np.abs(table), np.zeros(vocab, dtype=np.int64)
    for t, i in enumerate(ids):
        if 0 <= i < vocab:
            table[i] += scale * grad[t]
            size[i] += abs(scale) * np.abs(grad[t])
            terms[i] += 1
    return table, size, terms


def row_norm(h, weight, bias, eps, layer):
    n, _ = _normed(h, eps, layer)
    return n * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)


def _normed(h, eps, layer):
    c = h - h.mean(1, keepdims=True) if layer else h
    r = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    return c * r, r


def row_norm_backward(h, weight, eps, layer, grad, grad_sum=None):
    """(grad_h, what it is a sum of, grad_weight, its scale, grad_bias, its scale)."""
    n, r = _normed(h, eps, layer)
    g = grad * (1.0 if weight is None else weight)
    gh = g - n * (g * n).mean(1, keepdims=True)
    size = np.abs(g) + np.abs(n) * np.abs(g * n).mean(1, keepdims=True)
    if layer:
        gh = gh - g.mean(1, keepdims=True)
        size = size + np.abs(g).mean(1, keepdims=True)
    gh, size = r * gh, r * size
    if grad_sum is not None:
        gh, size = gh + grad_sum, size + np.abs(grad_sum)
    return gh, size, (grad * n).sum(0), np.abs(grad * n).sum(0), grad.sum(0), np.abs(grad).sum(0)


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-prob, number kept, margin) of one row; -1, nan, 0 where it has none. margin: how
    far, as a share of the masses, the nearest decision is from falling the other way."""
    bad = np.isnan(z).any() or (z == np.inf).any() or not (z > -np.inf).any()
    if bad or not 0.0 <= u <= 1.0 or not 0.0 <= temperature < np.inf or np.isnan(top_p) or np.isnan(min_p):
        return -1, np.nan, 0, 1.0
    order = np.nonzero(z > -np.inf)[0]
    order = order[np.lexsort((order, -z[order]))]
    if temperature == 0.0:
        return int(order[0]), 0.0, 1, 1.0
    t = (z[order] - z[order[0]]) / temperature
    w = np.exp(t)
    n, margin = len(order), 1.0
    if top_k > 0:
        n = min(n, top_k)
    c = np.cumsum(w)
    n_p = n_m = n
    if top_p < 1.0:
        want = top_p * c[n - 1]
        n_p = 1 + int((c[:n] < want).sum())
        margin = min(margin, float(np.min(np.abs(c[:n] - want)) / want)) if want > 0 else margin
    if min_p > 0.0:
        n_m = int((w >= min_p).sum())
        margin = min(margin, float(np.min(np.abs(w - min_p))) / min_p) if min_p != 1.0 else margin
    n = max(1, min(n, n_p, n_m))
    kept = np.sort(order[:n])
    wk = np.exp((z[kept] - z[order[0]]) / temperature)
    c = np.cumsum(wk)
    if u == 0.0 or u == 1.0:
        at = 0 if u == 0.0 else n - 1
    else:
        at = min(int((c <= u * c[-1]).sum()), n - 1)
        margin = min(margin, float(np.min(np.abs(c - u * c[-1])) / c[-1]))
    logp = (z[kept[at]] - z[order[0]]) / temperature - np.log(c[-1])
    return int(kept[at]), float(logp), n, margin
