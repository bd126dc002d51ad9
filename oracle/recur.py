"""Oracle of the gated linear recurrence (test infrastructure only): forward, gradients, and the magnitudes that
rounding errors are relative to.

Plain fp64 numpy, a loop over positions.  The paper has no counterpart (its Eq. 13 is the GRU whose linear form this is).
"""
import numpy as np


def gates(g, bias):
    """z and 1 - z, each from the exponential that does not cancel."""
    a = np.asarray(g, np.float64) + (0.0 if bias is None else bias)
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-a)), 1 / (1 + np.exp(a))


def forward(x, g, bias=None, lens=None, h_in=None):
    """x, g: n x T x d.  Returns y, the state after each sequence's last position, the states before each position, and
    the largest sum of absolute terms of a state of each sequence and channel (n x d)."""
    n, T, d = x.shape
    z, k = gates(g, bias)
    h = np.zeros((n, d)) if h_in is None else np.asarray(h_in, np.float64).copy()
    m = np.abs(h)
    most = m.copy()
    y, before = np.zeros((n, T, d)), np.zeros((n, T, d))
    for t in range(T):
        live = np.ones(n, bool) if lens is None else t < lens
        before[:, t] = h
        h[live] = k[live, t] * h[live] + z[live, t] * x[live, t]
        m[live] = k[live, t] * m[live] + z[live, t] * np.abs(x[live, t])
        y[live, t] = h[live]
        most = np.maximum(most, m)
    return y, h, before, most


def backward(x, g, dy, bias=None, lens=None, h_in=None, dh_out=None, held=False):
    """dx, dg, dbias, dh_in, and the same sums with every term's absolute value (x - h becomes |x| + the state's most);
    held: with R's most so far in the place of R's."""
    n, T, d = x.shape
    z, k = gates(g, bias)
    _, _, before, most = forward(x, g, bias, lens, h_in)
    R = np.zeros((n, d)) if dh_out is None else np.asarray(dh_out, np.float64).copy()
    own = np.abs(R)
    N = own.copy()
    out = {q: np.zeros((n, T, d)) for q in ("dx", "dg")}
    mag = {q: np.zeros((n, T, d)) for q in ("dx", "dg")}
    for t in reversed(range(T)):
        m = np.ones(n, bool) if lens is None else t < lens
        R[m] += dy[m, t]
        own[m] = own[m] + np.abs(dy[m, t])
        N[m] = np.maximum(N[m], own[m]) if held else own[m]
        out["dx"][m, t] = z[m, t] * R[m]
        mag["dx"][m, t] = z[m, t] * N[m]
        out["dg"][m, t] = R[m] * (x[m, t] - before[m, t]) * z[m, t] * k[m, t]
        mag["dg"][m, t] = N[m] * (np.abs(x[m, t]) + most[m]) * z[m, t] * k[m, t]
        R[m] *= k[m, t]
        own[m] *= k[m, t]
        N[m] = N[m] if held else own[m]
    for q, r in ((out, R), (mag, N)):
        q["dbias"], q["dh_in"] = q["dg"].sum((0, 1)), r
    return out, mag
