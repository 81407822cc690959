"""Filtered distributions, draws and the accept / resample rule from their definitions, in 64 bits (numpy)."""
import numpy as np


def f32(x):
    return float(np.float32(x))


class Row:
    """The filtered distribution of a row: probabilities p, and `margin`: how far (relative) the nearest border is from being moved by one id."""

    def __init__(self, z, T=1.0, top_k=0, top_p=0.0, min_p=0.0):
        z = np.asarray(z, dtype=np.float32).astype(np.float64) + 0.0
        T, top_p, min_p = f32(T), f32(top_p), f32(min_p)
        V = z.size
        self.p, self.margin = np.full(V, np.nan), np.inf
        self.fine = not np.any(np.isnan(z)) and np.isfinite(z.max())
        if not self.fine:
            return
        order = np.lexsort((np.arange(V), -z))
        order = order[z[order] > -np.inf]
        with np.errstate(under="ignore"):
            w = np.exp((z[order] - z.max()) / T)
        n = min(top_k, w.size) if top_k else w.size
        if 0.0 < top_p < 1.0:
            total = w[:n].sum()
            before = np.concatenate([[0.0], np.cumsum(w[:n])])[:n]
            self.margin = np.min(np.abs(before[1:] / (top_p * total) - 1.0)) if n > 1 else np.inf
            n = int(np.searchsorted(before, top_p * total, side="left"))
        if min_p:
            self.margin = min(self.margin, np.min(np.abs(w[1:] / min_p - 1.0)) if w.size > 1 else np.inf)
            n = min(n, int(np.count_nonzero(w >= min_p)))
        self.p = np.zeros(V)
        self.p[order[:n]] = w[:n] / w[:n].sum()
        self.order, self.n = order, n


def draw(w, u):
    """(first id whose cumulative weight exceeds u times the total, how far u is from a border)."""
    c = np.cumsum(w) / w.sum()
    u = f32(u)
    t = min(int(np.searchsorted(c, u, side="right")), w.size - 1)
    return t, float(min(abs(c[t] - u), abs(u - (c[t - 1] if t else 0.0)) if t else 1.0))


def verify(P, Q, draft, ua, ur, uf):
    """(n_accept, next token, ratios, smallest margin of the decisions) of Eq. 2 over final rows P and draft rows Q (Row)."""
    m = len(P)
    ratio, margin = np.zeros(m - 1), np.inf
    for k in range(m - 1):
        p, q = P[k].p[draft[k]], Q[k].p[draft[k]]
        ratio[k] = np.nan if not (P[k].fine and Q[k].fine) else 0.0 if p == 0 else np.inf if q == 0 else p / q
        margin = min(margin, P[k].margin, Q[k].margin)
        if not np.isnan(ratio[k]):
            margin = min(margin, abs(min(1.0, ratio[k]) - f32(ua[k])) if ratio[k] < 1.0 else np.inf)
        if not f32(ua[k]) < ratio[k]:
            if np.isnan(ratio[k]):
                return k, -1, ratio, margin
            rest = np.maximum(P[k].p - Q[k].p, 0.0)
            t, d = draw(rest if rest.sum() > 0 else P[k].p, ur[k])
            return k, t, ratio, min(margin, d)
    margin = min(margin, P[m - 1].margin)
    if not P[m - 1].fine:
        return m - 1, -1, ratio, margin
    t, d = draw(P[m - 1].p, uf)
    return m - 1, t, ratio, min(margin, d)
