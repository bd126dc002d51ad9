"""Oracle of the layer of experts (test infrastructure only): plain fp64 numpy, row after row.  The paper has no
counterpart."""
import numpy as np

from . import history as OH


def route(X, Wr, top, renorm, live=None):
    """Chosen experts (largest logit first, of equal ones the lower index) and their weights; -1 and 0 for a row that is
    not live."""
    n = len(X)
    idx, w = np.full((n, top), -1), np.zeros((n, top))
    for i in range(n):
        if live is not None and live[i] <= 0:
            continue
        l = X[i] @ Wr
        idx[i] = np.argsort(-l, kind="stable")[:top]
        p = np.exp(l - l.max())
        w[i] = p[idx[i]] / (p[idx[i]].sum() if renorm else p.sum())
    return idx, w


def forward(X, Wr, Wg, Wu, Wd, top, act, residual, renorm, live=None):
    """Y, experts, weights; and two sums of the absolute values of Y's terms: with the hidden rows as they are, and with
    the sums inside G and U taken by their absolute terms too."""
    idx, w = route(X, Wr, top, renorm, live)
    Y, rounded, terms = np.zeros_like(X), np.zeros_like(X), np.zeros_like(X)
    for i in range(len(X)):
        if live is not None and live[i] <= 0:
            continue
        if residual:
            Y[i] = X[i]
            terms[i] = np.abs(X[i])
        for e, s in zip(idx[i], w[i]):
            G, U = X[i] @ Wg[e], X[i] @ Wu[e]
            H = OH.act(G, act)[0] * U
            Y[i] += s * (H @ Wd[e])
            rounded[i] += s * (np.abs(H) @ np.abs(Wd[e]))
            terms[i] += s * (((np.abs(X[i]) @ np.abs(Wg[e])) * (np.abs(X[i]) @ np.abs(Wu[e]))) @ np.abs(Wd[e]))
    return Y, idx, w, rounded, terms
