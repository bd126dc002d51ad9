"""Edges of the history encoder's operators: values that are infinite, NaN or far from one, many rows a CTA, and bounds
as tight as the kernels' sums.  Helpers and the way tolerances are written: test_gpu_history.py."""
import numpy as np
import pytest
import torch

from hgsynth import bf16_round
from oracle import history as OH
from tests.gpu_util import dev, lib, need_gpu, tdtype
from tests.test_gpu_history import F32, U, f64, near, nans

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ gated block
GATES = np.array([0, 0.5, 2, 3.5, 7, 9, 20, 100, 300, 2.0**18, 1e6, 2.0**22, 1e10, 1e14, 1e20, 1e30], np.float32)


def gates_problem(dt):
    """G = the gates, U = 1, dH = dY: rows of gates in features 0..31 (feature 63 is one), unit weights."""
    vals = np.concatenate([GATES, -GATES])
    if dt == "bf16":
        vals = bf16_round(vals)
    n, d = 37, 64
    X, dY = np.zeros((n, d), np.float32), np.zeros((n, d), np.float32)
    X[:, :32] = vals[(np.arange(32) + np.arange(n)[:, None]) % 32]
    X[:, 63] = 1
    dY[:, :32] = np.where((np.arange(32) + np.arange(n)[:, None]) % 3 == 0, -0.75, 1.25)
    Wg, Wu, Wd = np.zeros((d, d), np.float32), np.zeros((d, d), np.float32), np.eye(d, dtype=np.float32)
    Wg[np.arange(32), np.arange(32)] = 1
    Wu[63] = 1
    return X, Wg, Wu, Wd, dY


def gates_run(hg, dt, act):
    """Y, dX and the weights' gradients of gates_problem, and what act and act' are there."""
    td = tdtype(dt)
    X, Wg, Wu, Wd, dY = gates_problem(dt)
    n, d = X.shape
    p = hg.FfnParams(*(dev(w, td) for w in (Wg, Wu, Wd)), act=act)
    work = torch.empty(max(hg.hg_ffn_workspace_size(p, n)), dtype=torch.uint8, device="cuda")
    Y, dX = nans((n, d), td), nans((n, d), td)
    g = {k: nans((d, d), torch.float32) for k in ("W_gate", "W_up", "W_down")}
    hg.hg_ffn_fwd(p, dev(X, td), Y, work)
    hg.hg_ffn_bwd(p, dev(X, td), dev(dY, td), dX, g, work)
    X, dY = f64(X), f64(dY)
    A, dA = OH.act(np.clip(X, -1e4, 1e4), act)
    if act != "none":  # beyond 1e4: x or 0, 1 or 0
        big = np.abs(X) > 1e4
        A, dA = np.where(big, np.maximum(X, 0), A), np.where(big, (X > 0) * 1.0, dA)
    else:
        A = X
    return X, dY, A, dA, Y, dX, g


g32 = slice(0, 32)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu", "none"])
def test_values_of_gates_of_every_size(dt, act):
    """act of gates from 0 to 1e30 of either sign.  G, U and dH are exact and a sum has one term: the functions within 30
    steps of |x|, in bf16 H rounded once; dW_up sums 37 rows, in bf16 of two terms."""
    need_gpu()
    X, dY, A, _, Y, _, g = gates_run(lib(), dt, act)
    near(Y[:, g32], A[:, g32], np.abs(X[:, g32]), (U[dt], 30 * F32), "Y")
    s = (2.0**-16 if dt == "bf16" else 0) + (30 + 37) * F32
    near(g["W_up"][63, g32], (dY * A).sum(0)[g32], (np.abs(dY) * np.abs(X)).sum(0)[g32], (0, s), "W_up")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu", "none"])
def test_derivatives_of_gates_of_every_size(dt, act):
    """act' of the same gates: that of a large one is 1 or 0.  Within 70 steps of 1 (a slope below 2.3 times 30 steps where
    it is neither 0 nor 1), in bf16 dG rounded once; dW_gate sums 37 rows, in bf16 of two terms."""
    need_gpu()
    X, dY, _, dA, _, dX, g = gates_run(lib(), dt, act)
    near(dX[:, g32], (dY * dA)[:, g32], np.abs(dY[:, g32]), (U[dt], 70 * F32), "dX")
    s = (2.0**-16 if dt == "bf16" else 0) + (70 + 37) * F32
    near(g["W_gate"][:, g32], X.T @ (dY * dA)[:, g32], np.abs(X).T @ np.abs(dY[:, g32]), (0, s), "W_gate")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "relu", "none"])
def test_a_gate_that_is_nan_is_seen(dt, act):
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    X, Wg, Wu, Wd, dY = gates_problem(dt)
    X[:, :32] = np.clip(X[:, :32], -4, 4)
    Wg[63, 40] = np.nan  # one hidden feature's gate, of every row
    n, d = X.shape
    p = hg.FfnParams(*(dev(w, td) for w in (Wg, Wu, Wd)), act=act)
    work = torch.empty(max(hg.hg_ffn_workspace_size(p, n)), dtype=torch.uint8, device="cuda")
    Y, dX = torch.zeros(n, d, dtype=td, device="cuda"), torch.zeros(n, d, dtype=td, device="cuda")
    g = {k: torch.zeros(d, d, device="cuda") for k in ("W_gate", "W_up", "W_down")}
    hg.hg_ffn_fwd(p, dev(X, td), Y, work)
    assert torch.isnan(Y).all()  # the feature is a term of every column
    dY[:, 40] = 1
    hg.hg_ffn_bwd(p, dev(X, td), dev(dY, td), dX, g, work)
    assert torch.isnan(dX).all() and torch.isnan(g["W_up"][:, 40]).all() and torch.isnan(g["W_down"][40]).all()
