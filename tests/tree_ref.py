"""Drafted trees, plainly: masks and positions node by node, verification as it is
defined (distributions that are subtracted and normalised again after each
rejection, in 64 bits), and the places that keeping a path copies."""
import numpy as np


def masks(parents, base, window=0):
    """(rows of booleans [n, n], positions [n]) of one sequence's nodes; what hangs on
    no earlier node sees nothing and has position -1."""
    n = len(parents)
    seen, pos = np.zeros((n, n), bool), np.full(n, -1, np.int64)
    for i in range(n):
        up, j = [], i
        while 0 <= j:
            up.append(j)
            p = int(parents[j])
            if p < -1 or p >= j:
                up = None
                break
            j = p
        if up is None:
            continue
        pos[i] = base + len(up) - 1
        seen[i, up[:window] if window else up] = True
    return seen, pos


def words(seen, n_words):
    """Rows of booleans as int32 words, bit j of word j / 32 first."""
    out = np.zeros((seen.shape[0], 32 * n_words), np.uint64)
    out[:, :seen.shape[1]] = seen[:, :32 * n_words]
    out = (out.reshape(-1, n_words, 32) << np.arange(32, dtype=np.uint64)).sum(axis=2)
    return out.astype(np.uint32).view(np.int32)


def softmax(x, temp):
    """Probabilities of a row of logits, or None where it has none."""
    x = np.asarray(x, np.float64)
    if np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
        return None
    live = x > -np.inf
    p = np.zeros(len(x))
    p[live] = np.exp((x[live] - x.max()) / temp)
    return p / p.sum()


def invert(w, u):
    """The first index at which the running sum of w passes u times the whole."""
    c = np.cumsum(w)
    return int(np.searchsorted(c, u * c[-1], side="right"))


def verify(parents, tokens, target, draft, random, temp=1.0, replace=False):
    """(path, next token) of one sequence.  draft: rows of logits, or None where the
    drafted tokens are points."""
    n = len(parents)
    u = np.nan_to_num(np.clip(np.asarray(random, np.float64), 0, 1 - 2.0 ** -24), nan=0.0)
    path, at = [0], 0
    while True:
        logits = np.asarray(target[at], np.float64)
        p = softmax(logits, temp if temp > 0 else 1.0)
        if p is None:
            return path, -1
        kids = [i for i in range(at + 1, n) if parents[i] == at]
        if not temp > 0:
            best = int(np.argmax(logits))  # the lowest of equals
            nxt = [i for i in kids if tokens[i] == best]
            if not nxt:
                return path, best
            at = nxt[0]
            path.append(at)
            continue
        q = None
        if draft is not None and kids:
            q = softmax(draft[at], temp)
            if q is None:
                return path, -1
        r, went, left = p, None, 1.0  # left: of p
        for i in kids:
            if left < 2.0 ** -32:
                break
            x = int(tokens[i])
            if not 0 <= x < len(p):
                continue
            if draft is None:
                if u[i] < r[x]:
                    went = i
                    break
                r = r.copy()
                r[x] = 0
            else:
                if u[i] * q[x] < r[x]:
                    went = i
                    break
                r = np.maximum(r - q, 0)
                if not replace:
                    q = q.copy()
                    q[x] = 0
                    if q.sum() > 0:
                        q = q / q.sum()
            left *= r.sum()
            if r.sum() > 0:
                r = r / r.sum()
        if went is None:
            return path, invert(r if left >= 2.0 ** -32 else p, u[0])
        at = went
        path.append(at)
