"""Sampling settings on rows of logits in plain numpy, for the sampling tests: values and
masses in 64 bits, sums of masses in 80 (a running sum of 33000 weights that each fall 1e-13 short of
1 loses all of that in 64 bits, where one step is 3.6e-12, and with it the place of a cut)."""
import numpy as np
import torch


def to64(t):
    return t.detach().cpu().double().numpy()


def kept(l, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Truth value for every element of the row l (float64): whether the settings keep it.
    None for a row without a distribution (a NaN, a +inf, no finite element)."""
    if np.isnan(l).any() or (l == np.inf).any() or not np.isfinite(l).any():
        return None
    T, top_p, min_p = (float(np.float32(x)) for x in (T, top_p, min_p))
    order = np.lexsort((np.arange(l.size), -l))
    order = order[np.isfinite(l[order])]
    w = np.exp((l[order] - l[order[0]]) / T).astype(np.longdouble)
    n = order.size if top_k == 0 else min(top_k, order.size)
    if top_p < 1.0:
        total = w[:n].cumsum()
        n = min(n, int((total < top_p * total[-1]).sum()) + 1)
    n = min(n, int((w >= min_p).sum()))
    mask = np.zeros(l.size, dtype=bool)
    mask[order[:n]] = True
    return mask


def draw(l, T, mask, u):
    """(token, log-probability) of the uniform u over the kept elements of the row l."""
    T = float(np.float32(T))
    a = (l - l[np.isfinite(l)].max()) / T
    w = np.where(mask, np.exp(a).astype(np.longdouble), 0.0)
    c = w.cumsum()
    j = int(np.searchsorted(c, float(np.float32(u)) * c[-1], side="right"))
    j = min(j, int(np.flatnonzero(w > 0.0)[-1]))
    return j, float(a[j] - np.log(c[-1]))


def border(l, T, mask, u):
    """How far u times the kept mass is from the nearest border between two tokens, over
    that mass."""
    T = float(np.float32(T))
    w = np.where(mask, np.exp((l - l[np.isfinite(l)].max()) / T).astype(np.longdouble), 0.0)
    c = w.cumsum()
    return np.abs(c - float(np.float32(u)) * c[-1]).min() / c[-1]


def logprob(l, T, token):
    """(log-probability, rank) of a token of the row l."""
    T = float(np.float32(T))
    a = (l - l[np.isfinite(l)].max()) / T
    before = (l > l[token]).sum() + (l[:token] == l[token]).sum()
    return a[token] - np.log(np.exp(a).sum()), 1 + int(before)


def make_rows(R, V, dtype, seed, kind="zipf", pad=0, offset=0, device="cuda"):
    """R rows of V logits on the GPU, `pad` elements of NaN after each, the first row `offset`
    elements into its memory."""
    g = np.random.default_rng([seed, R, V])
    if kind == "zipf":
        x = 5.0 - 1.1 * np.log(1.0 + V * g.random((R, V))) + 1.2 * g.standard_normal((R, V))
    elif kind == "flat":
        x = 0.01 * g.standard_normal((R, V))
    elif kind == "peaked":
        x = -4.0 + g.standard_normal((R, V))
        x[np.arange(R), g.integers(0, V, R)] += 30.0
    elif kind == "equal":
        x = np.full((R, V), -2.5)
    elif kind == "few":                    # a handful of distinct values, many ties
        x = g.integers(-3, 4, (R, V)) * 0.5
    elif kind == "masked":                 # most of the vocabulary masked with -inf
        x = g.standard_normal((R, V)) * 3.0
        x[g.random((R, V)) < 0.9] = -np.inf
        x[np.arange(R), g.integers(0, V, R)] = 1.0
    elif kind == "lowest":                 # masked with the type's lowest value
        x = g.standard_normal((R, V)) * 3.0
        x[g.random((R, V)) < 0.5] = torch.finfo(dtype).min
    elif kind == "all-lowest":
        x = np.full((R, V), torch.finfo(dtype).min)
    elif kind == "large":                  # far from zero
        x = 1.0e4 + 3.0 * g.standard_normal((R, V))
    else:
        raise ValueError(kind)
    flat = torch.full((offset + R * (V + pad),), float("nan"), dtype=dtype, device=device)
    rows = flat[offset:].view(R, V + pad)[:, :V]
    rows.copy_(torch.as_tensor(x, device=device).to(dtype))
    return rows
