"""Plain fp64 forms of the filtered sampler, the filtered row, the embedding lookup and its gradient, from their
definitions: sort by (logit descending, id ascending), three prefixes, inverse CDF in id order."""
import numpy as np

NONFINITE, FALLBACK, BAD_TEMPERATURE, BAD_FILTER = 4, 8, 32, 64


def kept_ids(z, part, tau, k, p, min_p):
    """(kept ids in id order, their weights, status) of one row; z float64 [V], part bool [V] (ids that take part)."""
    if not (tau >= 0 and np.isfinite(tau)):
        status = BAD_TEMPERATURE
    else:
        status = 0
    if np.isnan(p) or np.isnan(min_p):
        status |= BAD_FILTER
    if status:
        return None, None, status
    ids = np.flatnonzero(part)
    v = z[ids]
    if np.isnan(v).any() or (v == np.inf).any():
        return None, None, NONFINITE
    ids = ids[v > -np.inf]
    if ids.size == 0:
        return None, None, FALLBACK
    order = ids[np.argsort(-z[ids], kind="stable")]
    if tau == 0:
        return order[:1], np.ones(1), 0
    with np.errstate(over="ignore", under="ignore"):
        w = np.exp((z[order] - z[order[0]]) / float(tau))
    n = order.size if k <= 0 else min(int(k), order.size)
    order, w = order[:n], w[:n]
    c = np.cumsum(w)
    keep = np.ones(n, bool)
    if p < 1:
        keep &= np.concatenate(([0.0], c[:-1])) < float(p) * c[-1]
    if min_p > 0:
        keep &= w >= float(min_p)
    keep[0] = True
    ids = np.sort(order[keep])
    with np.errstate(over="ignore", under="ignore"):
        return ids, np.exp((z[ids] - z[order[0]]) / float(tau)), 0


def sample_row(ids, w, u):
    c = np.cumsum(w)
    above = np.flatnonzero(c > float(u) * c[-1])
    at = above[0] if above.size else np.flatnonzero(w > 0)[-1]
    return ids[at], w[at] / c[-1]


def rows(z, part, tau, k, p, min_p, u):
    """z float64 [B,R,V], part bool [V], the rest per sequence (u [B,R]): tokens, prob, status, kept mask."""
    B, R, V = z.shape
    tokens, prob = np.full((B, R), -1, np.int64), np.zeros((B, R))
    status, kept = np.zeros((B, R), np.int64), np.zeros((B, R, V), bool)
    for b in range(B):
        for r in range(R):
            ids, w, status[b, r] = kept_ids(z[b, r], part, tau[b], k[b], p[b], min_p[b])
            if ids is None:
                continue
            kept[b, r, ids] = True
            tokens[b, r], prob[b, r] = sample_row(ids, w, u[b, r])
    return tokens, prob, status, kept


def table_ids(ids, id_map, V_t, ids_side, table_side):
    """Ids carried to the table's vocabulary; sides 0 (target) and 1 (drafter)."""
    V_d = len(id_map)
    inv = np.full(V_t, -1, np.int64)
    inv[id_map[id_map >= 0]] = np.flatnonzero(id_map >= 0)
    ids = np.asarray(ids, np.int64)
    inside = (ids >= 0) & (ids < (V_d if ids_side else V_t))
    safe = np.where(inside, ids, 0)
    out = safe if ids_side == table_side else (id_map[safe] if ids_side else inv[safe])
    return np.where(inside, out, -1)
