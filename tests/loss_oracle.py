"""Plain fp64 forms of the losses and their gradients, row by row from the definitions."""
import numpy as np

NONFINITE, FALLBACK, BAD_TEMPERATURE, LEFT_OUT = 4, 8, 32, 128
MASK = -1e30


def targets(t, part, teacher, tau):
    """(ids that take part, their probabilities, |teacher - max|/tau) of one row; t [k] ids in the rows' vocabulary, -1 for none."""
    on = np.array([x >= 0 and part[x] for x in t])
    if teacher is not None:
        on &= ~(teacher < MASK)
    if not on.any():
        return None, None, None
    y = np.zeros(on.sum()) if teacher is None else teacher[on]
    if np.isnan(y).any() or (y == np.inf).any():
        return t[on], np.full(on.sum(), np.nan), None
    w = np.exp((y - y.max()) / tau)
    return t[on], w / w.sum(), np.where(y > -np.inf, y.max() - y, 0) / tau


def rows(z, part, t, teacher, tau):
    """z fp64 [N,V], part bool [V], t int [N,k], teacher fp64 [N,k] or None, tau [N] (float32 values).

    Returns loss, stats, status, q [N,V], p [N,V] (the targets' probabilities spread over the vocabulary), `terms` [N]: the
    size of what is added up beside ln(sum), and `far` [N,V]: the targets' |teacher - max|/tau weighed with their probabilities, spread alike."""
    N, V = z.shape
    loss, stats, status = np.zeros(N), np.zeros((N, 2)), np.zeros(N, np.int64)
    q, p, terms, far = np.zeros((N, V)), np.zeros((N, V)), np.zeros(N), np.zeros((N, V))
    for n in range(N):
        T = float(tau[n])
        with np.errstate(all="ignore"):
            s = np.float32(1.4426950408889634) / np.float32(T)
        bad_tau = not (T > 0 and np.isfinite(T) and s > 0 and np.isfinite(s))
        ids, prob, gap = targets(t[n], part, None if teacher is None else teacher[n], 1.0 if bad_tau else T)
        if ids is None or bad_tau:
            status[n] = (LEFT_OUT if ids is None else 0) | (BAD_TEMPERATURE if bad_tau else 0)
            continue
        y = np.where(part, z[n], -np.inf)
        y = np.where(y < MASK, -np.inf, y)
        if np.isnan(y).any() or (y == np.inf).any() or np.isnan(prob).any():
            status[n], loss[n], q[n] = NONFINITE, np.nan, np.nan
            stats[n] = (np.nan, np.nan)
            continue
        if (y == -np.inf).all():
            status[n] = FALLBACK
            continue
        m = y.max()
        w = np.exp((y - m) / T)
        stats[n] = m, w.sum()
        q[n] = w / w.sum()
        np.add.at(p[n], ids, prob)
        np.add.at(far[n], ids, prob * gap)
        with np.errstate(divide="ignore"):
            up = prob > 0
            each = prob[up] * (np.log(prob[up]) + (m - y[ids[up]]) / T)
            terms[n] = (prob[up] * (np.abs(np.log(prob[up])) + (m - y[ids[up]]) / T)).sum()
        loss[n] = np.log(w.sum()) + each.sum()
    return loss, stats, status, q, p, terms, far
