"""Oracle of the history encoder's operators (test infrastructure only): norm and rotation of query and key
heads, linear attention with a decay for each head, gated feed-forward block, and their gradients.

Plain fp64 numpy from the formulas; each sum is written where the formula has it (a loop over positions for
the recurrence).  The paper has no counterpart.  `magnitude` forms sum the absolute values of the same terms:
what a rounding of the terms is relative to.
"""
import numpy as np


# ---------------------------------------------------------------------------------------------- rotation
def angles(pos, rot, base):
    """pos * base^(-2 i / rot), i < rot / 2 (n x rot / 2)."""
    return np.asarray(pos, np.float64)[:, None] * np.float64(base) ** (-2.0 * np.arange(rot // 2) / max(rot, 1))


def pair_index(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turn(y, ang, rot, interleaved):
    a, b = pair_index(rot, interleaved)
    out = y.copy()
    c, s = np.cos(ang)[:, None, :], np.sin(ang)[:, None, :]
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    return out


def qkrot_forward(x, gamma, pos, rot, base, eps, interleaved):
    """x: n x heads x d_h."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return turn(x * r * gamma, angles(pos, rot, base), rot, interleaved)


def qkrot_backward(x, gamma, pos, rot, base, eps, interleaved, dy):
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = x * r
    g = turn(dy, -angles(pos, rot, base), rot, interleaved)
    c = g * gamma
    return r * (c - u * (c * u).mean(-1, keepdims=True)), (g * u).sum((0, 1))


# ------------------------------------------------------------------------------------------------- decay
def decay_forward(q, k, v, log_decay, scale, lens=None, S_in=None, magnitude=False):
    """q, k, v: n x T x heads x d_h.  Returns o and the state after each sequence's last position."""
    n, T, h, d = q.shape
    f = np.abs if magnitude else (lambda x: x)
    gamma = np.exp(np.minimum(log_decay, 0.0))[:, None, None]
    S = np.zeros((n, h, d, d)) if S_in is None else f(S_in).copy()
    o = np.zeros((n, T, h, d))
    for t in range(T):
        live = np.ones(n, bool) if lens is None else t < lens
        new = gamma * S[live] + f(k[live, t])[..., :, None] * f(v[live, t])[..., None, :]
        S[live] = new
        o[live, t] = scale * np.einsum("nhi,nhij->nhj", f(q[live, t]), new)
    return o, S


def decay_backward(q, k, v, log_decay, scale, do, lens=None, S_in=None, dS_out=None, magnitude=False):
    n, T, h, d = q.shape
    f = np.abs if magnitude else (lambda x: x)
    gamma = np.exp(np.minimum(log_decay, 0.0))[:, None, None]
    S = np.zeros((n, h, d, d)) if S_in is None else f(S_in).copy()
    R = np.zeros((n, h, d, d)) if dS_out is None else f(dS_out).copy()
    dq, dk, dv = (np.zeros((n, T, h, d)) for _ in range(3))
    alive = lambda t: np.ones(n, bool) if lens is None else t < lens  # noqa: E731
    for t in range(T):
        m = alive(t)
        S[m] = gamma * S[m] + f(k[m, t])[..., :, None] * f(v[m, t])[..., None, :]
        dq[m, t] = scale * np.einsum("nhij,nhj->nhi", S[m], f(do[m, t]))
    for t in reversed(range(T)):
        m = alive(t)
        now = R[m] + scale * f(q[m, t])[..., :, None] * f(do[m, t])[..., None, :]
        dk[m, t] = np.einsum("nhij,nhj->nhi", now, f(v[m, t]))
        dv[m, t] = np.einsum("nhi,nhij->nhj", f(k[m, t]), now)
        R[m] = gamma * now
    return dq, dk, dv, R


# ------------------------------------------------------------------------------------------------ gated block
def act(g, kind):
    """act(g) and its derivative."""
    if kind == "relu":
        return np.maximum(g, 0.0), (g > 0).astype(np.float64)
    if kind == "none":
        return g, np.ones_like(g)
    if kind == "silu":
        z, dz = g, np.ones_like(g)
    else:  # (1 + tanh(z / 2)) / 2 = 1 / (1 + e^-z)
        c = 2 * np.sqrt(2 / np.pi)
        z, dz = c * (g + 0.044715 * g ** 3), c * (1 + 3 * 0.044715 * g * g)
    e = np.exp(-np.abs(z))
    s = np.where(z >= 0, 1 / (1 + e), e / (1 + e))
    return g * s, s + g * dz * e / (1 + e) ** 2


def ffn_forward(X, Wg, Wu, Wd, kind, residual):
    y = (act(X @ Wg, kind)[0] * (X @ Wu)) @ Wd
    return y + X if residual else y


def ffn_backward(X, Wg, Wu, Wd, kind, residual, dY):
    """dX, dW_gate, dW_up, dW_down."""
    U, dH = X @ Wu, dY @ Wd.T
    A, dA = act(X @ Wg, kind)
    dG, dU = dH * U * dA, dH * A
    dX = dG @ Wg.T + dU @ Wu.T
    return (dX + dY if residual else dX), X.T @ dG, X.T @ dU, (A * U).T @ dY
