"""A plain implementation of beam search's selection: numpy in 64 bits, written from the contract."""
import math

import numpy as np


def log_softmax(row):
    l = np.where(np.isnan(row), -math.inf, row.astype(np.float64))
    top = l.max()
    if top == -math.inf:
        return l, l
    with np.errstate(invalid="ignore"):
        x = np.where(l == top, 0.0, l - top)
    return l, x - math.log(math.fsum(np.exp(x[x > -745])))


def select(logits, scores, n, finished=None, end_token=0, norm=None):
    """One sentence: logits [K, V], scores [K]: ([(score, parent, token)], least distance of neighbouring ranks of different beams among the n + 1 best)."""
    found = []
    for k in range(len(scores)):
        if not scores[k] > -math.inf:
            continue
        f = 1.0 if norm is None else float(norm[k])
        if finished is not None and finished[k]:
            found.append((float(scores[k]) * f, k, 0, float(scores[k]), end_token))
            continue
        l, logp = log_softmax(logits[k])
        order = np.lexsort((np.arange(len(l)), -l))[:n + 1]
        for j, v in enumerate(order):
            s = float(scores[k]) + logp[v]
            if s > -math.inf:
                found.append((s * f, k, j, s, int(v)))
    found.sort(key=lambda c: (-c[0], c[1], c[2]))
    near = min([a[0] - b[0] for a, b in zip(found[:n], found[1:n + 1]) if a[1] != b[1]], default=math.inf)
    best = [(c[3], c[1], c[4]) for c in found[:n]]
    return best + [(-math.inf, -1, -1)] * (n - len(best)), near
