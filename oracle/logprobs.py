"""Oracle: log-probabilities of given tokens through the LM head, entropies and top alternatives.

Test infrastructure only: the GPU library never imports this module.

z = h W^T, lse = log sum exp z, logp = z_y - lse, entropy = -sum p log p with p = softmax(z) (a term of p = 0 is 0);
the alternatives are the largest z, equal ones in the order of their ids. A label outside [0, V)
has logp NaN. A row whose lse is not finite has NaN everywhere and the ids -1. float64.
"""
import numpy as np


def token_logprobs(h, W, labels, top):
    """dict(logp, entropy [N], ids, top [N, top], size): size [N] is the largest sum |h||w| of a row's logits."""
    h, W = np.asarray(h, np.float64), np.asarray(W, np.float64)
    N, V = h.shape[0], W.shape[0]
    with np.errstate(all="ignore"):
        z = h @ W.T
        size = (np.abs(h) @ np.abs(W).T).max(1)
        m = z.max(1, keepdims=True)
        e = np.exp(z - m)
        lse = m + np.log(e.sum(1, keepdims=True))
        lp = z - lse
        p = np.exp(lp)
        entropy = -np.where(p > 0, p * lp, np.where(np.isnan(p), np.nan, 0.0)).sum(1)
        inside = (labels >= 0) & (labels < V)
        logp = np.where(inside, lp[np.arange(N), np.where(inside, labels, 0)], np.nan)
        ids = np.argsort(-z, axis=1, kind="stable")[:, :top]
    fine = np.isfinite(lse[:, 0])
    logp, entropy = np.where(fine, logp, np.nan), np.where(fine, entropy, np.nan)
    best = np.where(fine[:, None], np.take_along_axis(lp, ids, 1), np.nan)
    return dict(logp=logp, entropy=entropy, ids=np.where(fine[:, None], ids, -1).astype(np.int32), top=best, size=size)
