"""Log probabilities, ranks, entropy and order of the tokens of rows of logits in fp64, from their definitions (include/blink.h). Oracle
code: test infrastructure only."""
import numpy as np


def row(x, inverse=1.0):
    """x [vocab] -> dict(logp [vocab], entropy, order [vocab] (ids, first to last), p [vocab], z - max [vocab])."""
    x = np.asarray(x, dtype=np.float64)
    order = np.lexsort((np.arange(x.size), -np.where(np.isnan(x), -np.inf, x)))
    with np.errstate(all="ignore"):
        if not (inverse > 0 and np.isfinite(inverse)):
            inverse = np.nan
        d = (x - x.max()) * inverse                     # (NaN if there is one, or nothing but -inf)
        e = np.exp(d)
        logp = d - np.log(e.sum())
        p = np.exp(logp)
        entropy = -np.where(p > 0, p * logp, p * 0).sum()
    return dict(logp=logp, entropy=entropy, order=order, p=p, d=d)


def ranks(r, tokens):
    """Places of tokens in the order; -1: outside the vocabulary."""
    place = np.empty(r["order"].size, dtype=np.int64)
    place[r["order"]] = np.arange(place.size)
    return np.array([place[t] if 0 <= t < place.size else -1 for t in tokens])
