"""The definition of octopus_verify_drafts for one sequence, in extended precision (64-bit sums that err by less than u's 24 bits can tell
would do; these keep eleven bits more)."""
import numpy as np


def counted(p):
    p = np.asarray(p, dtype=np.float32).astype(np.float64)
    return np.where((p > 0) & np.isfinite(p), p, 0.0)


def inside(u):
    u = np.float32(u)
    return float(min(u, np.float32(1 - 2 ** -24))) if u > 0 else 0.0


def verify(target, draft, x, u, n_draft):
    """target [n + 1, vocab], draft [n, vocab] or None, x [n] -> (tokens [n_draft + 1], drafts that stand)"""
    n, vocab = len(x), target.shape[1]
    a = 0
    for i in range(n):
        if not 0 <= x[i] < vocab:
            break
        q = 1.0 if draft is None else counted(draft[i])[x[i]]
        if not inside(u[i]) * q < counted(target[i])[x[i]]:
            break
        a += 1
    p = counted(target[a])
    rest = p.copy()
    if a < n and draft is not None:
        rest = np.maximum(p - counted(draft[a]), 0.0)
    elif a < n and 0 <= x[a] < vocab:
        rest[x[a]] = 0.0
    if not np.any(rest > 0):
        rest = p
    token = -1
    at = np.nonzero(rest > 0)[0]
    if len(at):
        upto = np.cumsum(rest[at].astype(np.longdouble))
        goal = np.longdouble(inside(u[n_draft])) * upto[-1]
        token = int(at[min(np.searchsorted(upto, goal, side="right"), len(at) - 1)])
    return [int(t) for t in x[:a]] + [token] + [-1] * (n_draft - a), a
