"""Sampling and acceptance at temperature > 0 from their definition, in numpy doubles, one row at a time."""
import numpy as np


def kept_weights(l, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Weight of every token of the row l, 0 where it is not kept."""
    l = np.asarray(l, np.float32).astype(np.float64)
    V = len(l)
    out = np.zeros(V)
    ranking = [i for i in np.lexsort((np.arange(V), -np.where(np.isnan(l), -np.inf, l) + 0.0)) if not np.isnan(l[i])]
    if not ranking:
        return out
    ranking = np.array(ranking)
    if not temperature > 0 or l[ranking[0]] == -np.inf:
        out[ranking[0]] = 1.0
        return out
    t = min(np.float64(np.float32(temperature)), np.float64(np.finfo(np.float32).max))
    top = l[ranking[0]]
    kept = ranking[:top_k] if top_k > 0 else ranking
    with np.errstate(invalid="ignore"):
        w = np.where(l[kept] == top, 1.0, np.exp((l[kept] - top) / t))
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        n = max(1, int((before < np.float64(np.float32(top_p)) * w.sum()).sum()))
        kept, w = kept[:n], w[:n]
    if min_p > 0:
        n = max(1, int((w >= np.float64(np.float32(min_p))).sum()))
        kept, w = kept[:n], w[:n]
    out[kept] = w
    return out


def draw(w, u):
    """The first index whose running weight exceeds u of the whole (u outside [0, 1): the nearest border, NaN: the upper)."""
    c = np.cumsum(w)
    if not c[-1] > 0:
        return 0
    u = 1.0 if np.isnan(u) else float(np.float32(u))
    over = np.nonzero((c > u * c[-1]) & (w > 0))[0]
    return int(over[0]) if len(over) else int(np.nonzero(w > 0)[0][-1])


def near_border(w, u, ids):
    """ids draws no token of weight 0, and lies where u falls if every weight and partial sum may be off by its roundings: a
    weight by 4 half steps of a double, a sum of n of them by n more."""
    c, n = np.cumsum(w), len(w)
    u = 1.0 if np.isnan(u) else min(max(float(np.float32(u)), 0.0), 1.0)
    slack = (n + 8) * 2.0 ** -53 * c[-1]
    return w[ids] > 0 and c[ids] > u * c[-1] - slack - (u >= 1) * c[-1] * 2.0 ** -52 and c[ids] - w[ids] <= u * c[-1] + slack


def accept(draft, target, u_accept, u_sample, settings, draft_weights=None):
    """One sequence: (accepted slots, drawn token, what it was drawn from)."""
    k, V = len(draft), target.shape[1]
    for i in range(k + 1):
        p = kept_weights(target[i], *settings)
        p = p / p.sum() if p.sum() > 0 else p
        if i == k:
            return i, draw(p, u_sample), p
        d = int(draft[i])
        q = np.zeros(V)
        if draft_weights is not None:
            q = draft_weights[i] / max(draft_weights[i].sum(), 5e-324)
        elif 0 <= d < V:
            q[d] = 1.0
        if 0 <= d < V and float(np.float32(u_accept[i])) * q[d] < p[d]:
            continue
        rest = np.maximum(p - q, 0.0)
        if not rest.sum() > 0:
            rest = p
        return i, draw(rest, u_sample), rest
